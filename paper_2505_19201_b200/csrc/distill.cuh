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
#define DISTILL_THREADS 256
#define DISTILL_MAX_CLUSTER 8
#define DISTILL_MAX_VOCAB 262144

struct DistillArgs {
  const void *logits;
  long long ld;
  int vocab, cluster, cta_vecs, top;
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
__device__ __forceinline__ int teacher_warps(const DistillArgs &a) { return (a.top + 31) >> 5; }
struct TeacherRow {
  double f[DISTILL_TOP_WARPS];         // q_j = e_j f of its warp
  double rest, total, ref, sum;        // q_r; Q; without teacher_lse sum q ln q = (sum of f log) - ref - ln sum
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
// By the first teacher_warps() warps.
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
  const int n = teacher_warps(a);
#pragma unroll
  for (int w = 0; w < DISTILL_TOP_WARPS; ++w)
    if (!a.teacher_lse && w < n) m = fmax(m, sh.ref[w]);
#pragma unroll
  for (int w = 0; w < DISTILL_TOP_WARPS; ++w) {
    r.f[w] = w < n ? 1.0 : 0.0;
    if (!a.teacher_lse && w < n && sh.ref[w] != m) r.f[w] = sh.ref[w] > -INFINITY ? exp(sh.ref[w] - m) : 0.0;
    if (w < n) s += sh.sum[w] * r.f[w];
  }
  const bool any = !(s == 0.0);                             // a row with no valid entry has no loss, with or without the rest
  if (a.teacher_lse) {
    r.rest = any ? fmax(0.0, 1.0 - s) : 0.0;
    r.total = any ? s + r.rest : 0.0;
    r.ref = 0.0; r.sum = 1.0;
  } else {
#pragma unroll
    for (int w = 0; w < DISTILL_TOP_WARPS; ++w) r.f[w] = any ? r.f[w] / s : 0.0;
    r.rest = 0.0;
    r.total = any ? 1.0 : 0.0;
    r.ref = any ? m : 0.0; r.sum = any ? s : 1.0;
  }
  return r;
}

// A CTA's part in the row's sums, which are of 2^((l - m) ch), ch = log2(e) / tau.  (l ch - m ch in one instruction would overflow on rows
// masked with the type's lowest value.)
struct DistillPart {
  float m, unused;                     // largest logit, -inf without one
  double others, tops, qz;             // sums over the ids that are not listed, that are; sum of q_j z_j tau
};
#define DISTILL_PAIRS (DISTILL_THREADS / 32 + DISTILL_TOP_WARPS)
struct DistillShared {
  DistillPart part[DISTILL_MAX_CLUSTER];
  TeacherSums teacher;
  double q[DISTILL_MAX_TOP], qz[DISTILL_TOP_WARPS], qz_row, entropy;
  float2 pair[DISTILL_PAIRS];          // (maximum, sum): of every warp's vectors, of its listed ids
  float total, rest;                   // Q, q_r
  int id[DISTILL_MAX_TOP], repeated;
};
// Shared memory behind it: a byte per vector of the CTA's share, whose bits say which ids are listed, 16 bytes of such bits for the ids
// at the row's ends, then the vectors.
__host__ __device__ inline int distill_flag_bytes(int cta_vecs) { return (cta_vecs + 15) / 16 * 16 + 16; }

__device__ __forceinline__ void cp_async16(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A CTA's share of a row: whole vectors of 16 bytes on 16-byte boundaries, whatever the row's own alignment, thread t having the vectors t,
// t + threads, ..; and of the fewer than 2 VEC ids in front of the row's first boundary and behind its last, one for a thread at most.
template <typename T> struct RowShare {
  static constexpr int VEC = 16 / sizeof(T);
  const T *row, *mine;                 // the row; the thread's first vector
  int id0, nv, edge;                   // id of the share's first whole vector, how many there are, the thread's single id or -1
  __device__ __forceinline__ RowShare(const void *p, long long ld, int r, int vocab, int rank, int cluster, int cta_vecs) {
    row = (const T *)p + r * ld;
    const int tid = threadIdx.x, head = min(vocab, (VEC - (int)((uintptr_t)row / sizeof(T) % VEC)) % VEC), all = (vocab - head) / VEC,
              rest = vocab - head - all * VEC, v0 = min(all, rank * cta_vecs);
    id0 = head + v0 * VEC;
    nv = min(cta_vecs, all - v0);
    mine = row + id0 + tid * VEC;
    edge = rank == 0 && tid < head ? tid : rank == cluster - 1 && tid >= 16 && tid < 16 + rest ? vocab - rest + tid - 16 : -1;
  }
  // Where a listed id is in the share: a bit of a byte per vector, or of the bytes of the edges behind them; -1 elsewhere.
  __device__ __forceinline__ int flag_bit(int id, int vocab, int rank, int cluster) const {
    const int at = id - id0;
    if (id < 0) return -1;
    if (at >= 0 && at < nv * VEC) return at / VEC * 8 + at % VEC;
    const int n = flag_bytes(nv) * 8;
    if (at < 0) return rank == 0 && id0 < VEC ? n + id : -1;                          // in front of the first boundary
    return rank == cluster - 1 ? n + 16 + at - nv * VEC : -1;                         // behind the last
  }
  __host__ __device__ static int flag_bytes(int nv) { return (nv + 15) / 16 * 16; }
};

// The gradient coef * 2^((l - ref) ch - d) of the thread's vectors, get(k) being the k-th's logits, and of its single id's logit le (where
// `edge`).  Nothing is got where it is zero.  listed(g): bits of the elements of vector g that somebody else writes.
template <typename T, typename F, typename L>
__device__ __forceinline__ void write_row(const RowShare<T> &sr, T *dst, bool zero, F get, L listed, bool edge, float le, float ref, float ch, float d, float coef) {
  constexpr int VEC = 16 / sizeof(T), NT = DISTILL_THREADS;
  const float2 r2 = make_float2(-ref, -ref), c2 = make_float2(ch, ch), d2 = make_float2(-d, -d), o2 = make_float2(coef, coef);
  T *p = dst + sr.id0 + threadIdx.x * VEC;
  const bool vec = ((uintptr_t)p & 15) == 0;
  if (edge) dst[sr.edge] = from_f<T>(zero ? 0.f : coef * ex2(fmaf(le - ref, ch, -d)));
  for (int k = 0, g = threadIdx.x; g < sr.nv; ++k, g += NT, p += NT * VEC) {
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    if (!zero) {
      float l[VEC];
      unpack_vec<T, VEC>(get(k), l);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = fma_pair(add_pair(make_float2(l[e], l[e + 1]), r2), c2, d2);
        const float2 o = mul_pair(make_float2(ex2(y.x), ex2(y.y)), o2);
        l[e] = o.x; l[e + 1] = o.y;
      }
      q = pack_vec<T, VEC>(l);
    }
    const uint32_t not_mine = listed(g);
    if (vec && !not_mine) *reinterpret_cast<uint4 *>(p) = q;
    else {
      T u[VEC];
      memcpy(u, &q, 16);
#pragma unroll
      for (int e = 0; e < VEC; ++e) if (!(not_mine >> e & 1u)) p[e] = u[e];
    }
  }
}

// A thread has the same vectors of the share in every pass over it, so its copies into shared memory need no barrier: DISTILL_RING of them are
// on their way at a time, in groups of DISTILL_BATCH.  GRAD: the whole share stays there and its gradient leaves in the same call.
#define DISTILL_RING 16
#define DISTILL_BATCH 2
#define DISTILL_GRAD_RING 8
template <typename T, bool GRAD>
__global__ void __launch_bounds__(DISTILL_THREADS, 3)
k_distill(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillShared &sh = *reinterpret_cast<DistillShared *>(smem_raw);
  uint8_t *flags = smem_raw + (sizeof(DistillShared) + 15) / 16 * 16;
  constexpr int VEC = 16 / sizeof(T), NT = DISTILL_THREADS, NW = NT / 32, B = DISTILL_BATCH, AHEAD = DISTILL_RING / B;
  cluster_started_arrive(a.cluster);
  kernel_entry(TR_k_distill);
  const int rank = a.cluster > 1 ? (int)cluster_ctarank() : 0, row = blockIdx.x / a.cluster, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const RowShare<T> sr(a.logits, a.ld, row, a.vocab, rank, a.cluster, a.cta_vecs);
  uint4 *vals = reinterpret_cast<uint4 *>(flags + distill_flag_bytes(a.cta_vecs)) + tid;
  const float ch = (float)(a.inv_tau * 1.4426950408889634);
  const bool tail = a.teacher_lse != nullptr, top_warp = warp < teacher_warps(a);
  const int nb = (sr.nv + B * NT - 1) / (B * NT);           // batches
  for (int b = 0; b < (GRAD ? max(nb, AHEAD) : AHEAD); ++b) {
#pragma unroll
    for (int k = 0; k < B; ++k)
      if ((b * B + k) * NT + tid < sr.nv) cp_async16(vals + (b * B + k) * NT, sr.mine + (size_t)(b * B + k) * NT * VEC);
    cp_async_commit();
  }
  // while they are on their way: the teacher's side, and the listed ids' logits
  Entry t = {-1, -INFINITY, 0.0};
  if (top_warp) { t = load_entry(a, row); sh.id[tid] = t.id; }
  const float le = sr.edge >= 0 ? to_f(sr.row[sr.edge]) : -INFINITY, rs = GRAD && a.row_scale ? a.row_scale[row] : 1.f;
  for (int i = tid; i < distill_flag_bytes(sr.nv) / 4; i += NT) reinterpret_cast<uint32_t *>(flags)[i] = 0;
  if (tid == 0) sh.repeated = 0;
  if (tid < DISTILL_TOP_WARPS) sh.pair[NW + tid] = make_float2(-INFINITY, 0.f);
  const int bit = top_warp ? sr.flag_bit(t.id, a.vocab, rank, a.cluster) : -1;
  const bool mine = bit >= 0;
  const float z = mine ? to_f(sr.row[t.id]) : -INFINITY;
  __syncthreads();
  bool first = mine;                                        // of the entries of one id the first stands for it
  auto listed_pair = [&]() {
    const float tm = warp_max(z), ts = warp_sum(first ? ex2((z - (tm > -INFINITY ? tm : 0.f)) * ch) : 0.f);
    if (lane == 0) sh.pair[NW + warp] = make_float2(tm, ts);
  };
  if (top_warp) {
    if (mine && (atomicOr(reinterpret_cast<uint32_t *>(flags) + (bit >> 5), 1u << (bit & 31)) >> (bit & 31) & 1u)) sh.repeated = 1;
    teacher_sums(a, row, t, sh.teacher);
    const double qz = warp_sum_d(mine && !(t.e == 0.0) ? t.e * (double)z : 0.0);
    if (lane == 0) sh.qz[warp] = qz;
    listed_pair();
  }
  __syncthreads();
  TeacherRow tr;
  double qj = 0.0;
  if (top_warp) {
    tr = teacher_row(a, sh.teacher);
    sh.q[tid] = qj = t.e * tr.mine();
    if (sh.repeated) {
      for (int j = 0; j < tid; ++j) if (sh.id[j] == t.id) first = false;
      listed_pair();
    }
    if (tid == 0) {
      double qz = 0.0, en = -(tr.ref + log(tr.sum));        // sum q ln q, the bucket's too
      for (int w = 0; w < teacher_warps(a); ++w) {
        if (!(sh.qz[w] == 0.0)) qz += sh.qz[w] * tr.f[w];
        if (!(sh.teacher.log[w] == 0.0)) en += sh.teacher.log[w] * tr.f[w];
      }
      if (tr.rest > 0.0) en += tr.rest * log(tr.rest);
      sh.qz_row = qz; sh.entropy = en;
      sh.total = (float)tr.total; sh.rest = (float)tr.rest;
    }
  }
  // running maximum m (ref: the same, 0 without one) and sum of 2^((l - ref) ch); listed ids stay out where the rest is a bucket
  float m = -INFINITY, ref = 0.f, s = 0.f, s1 = 0.f;
  const bool listed_edge = sr.edge >= 0 && (flags[RowShare<T>::flag_bytes(sr.nv) + (tid >> 3)] >> (tid & 7) & 1u);
  if (sr.edge >= 0 && !(tail && listed_edge)) {
    if (le > m) { m = ref = le; s = 1.f; }
    else if (le != le) s = le;
  }
  for (int b = 0; b < nb; ++b) {
    cp_async_wait<AHEAD - 1>();
    uint4 q[B];
    uint32_t listed = 0;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const int g = (b * B + k) * NT + tid, slot = GRAD ? b * B + k : b % AHEAD * B + k;
      if (g < sr.nv) {
        q[k] = vals[slot * NT];
        if (tail) listed |= (uint32_t)flags[g] << k * VEC;
      } else {
        const uint32_t u = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;       // -inf
        q[k] = make_uint4(u, u, u, u);
      }
      if (!GRAD && g + DISTILL_RING * NT < sr.nv) cp_async16(vals + slot * NT, sr.mine + (size_t)((b + AHEAD) * B + k) * NT * VEC);
    }
    cp_async_commit();
    float l[B][VEC], v = max_vec<T, VEC>(q[0]);
#pragma unroll
    for (int k = 0; k < B; ++k) unpack_vec<T, VEC>(q[k], l[k]);
#pragma unroll
    for (int k = 1; k < B; ++k) v = fmaxf(v, max_vec<T, VEC>(q[k]));
    if (listed) {
      v = -INFINITY;
#pragma unroll
      for (int e = 0; e < B * VEC; ++e) {
        if (listed >> e & 1u) l[e / VEC][e % VEC] = -INFINITY;
        v = fmaxf(v, l[e / VEC][e % VEC]);
      }
    }
    if (v > m) {
      if (m > -INFINITY) { const float f = ex2((m - v) * ch); s *= f; s1 *= f; }
      m = ref = v;
    }
    const float2 r2 = make_float2(-ref, -ref), c2 = make_float2(ch, ch);
#pragma unroll
    for (int k = 0; k < B; ++k)
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = mul_pair(add_pair(make_float2(l[k][e], l[k][e + 1]), r2), c2);
        s += ex2(y.x); s1 += ex2(y.y);
      }
  }
  {
    const float wm = warp_max(m);
    s = warp_sum((s + s1) * (m > -INFINITY ? ex2((m - wm) * ch) : 1.f));        // without a maximum 0, or NaN
    if (lane == 0) sh.pair[warp] = make_float2(wm, s);
  }
  __syncthreads();
  // the CTA's sums out of the warps' (each thread that needs them by itself), in the precision asked for
  float rm = -INFINITY;
#pragma unroll
  for (int w = 0; w < DISTILL_PAIRS; ++w) rm = fmaxf(rm, sh.pair[w].x);
  auto join = [&](auto &others, auto &tops) {
#pragma unroll
    for (int w = 0; w < DISTILL_PAIRS; ++w) {
      const float2 p = sh.pair[w];
      const float v = p.x > -INFINITY ? p.y * ex2((p.x - rm) * ch) : p.y;
      if (w < NW) others += v;
      else if (tail) tops += v;                             // without the bucket they are among the others
    }
  };
  auto join_parts = [&](auto &others, auto &tops, double &qz) {
    for (int c = 0; c < a.cluster; ++c) {
      const DistillPart &p = sh.part[c];
      const float f = p.m > -INFINITY ? ex2((p.m - rm) * ch) : 1.f;
      others += p.others * f; tops += p.tops * f; qz += p.qz;
    }
  };
  if (a.cluster > 1) {
    cluster_started_wait(a.cluster);
    if (tid < a.cluster) {
      double others = 0.0, tops = 0.0;
      join(others, tops);
      const uint32_t to = mapa(smem_u32(&sh.part[rank]), tid);
      st_cluster_u64(to, (unsigned long long)__float_as_uint(rm));
      st_cluster_u64(to + 8, __double_as_longlong(others));
      st_cluster_u64(to + 16, __double_as_longlong(tops));
      st_cluster_u64(to + 24, __double_as_longlong(sh.qz_row));
    }
    cluster_sync_all();
    for (int c = 0; c < a.cluster; ++c) rm = fmaxf(rm, sh.part[c].m);
  }
  if (GRAD) {
    float others = 0.f, tops = 0.f;
    double unused = 0.0;
    if (a.cluster > 1) join_parts(others, tops, unused);
    else join(others, tops);
    const float total = others + tops, ref = rm > -INFINITY ? rm : 0.f, d = __log2f(total), scale = total == 0.f || sh.total == 0.f ? 0.f : rs * (float)a.inv_tau,
                coef = scale * (sh.total - (sh.rest > 0.f && others > 0.f ? sh.rest * __fdividef(total, others) : 0.f));
    T *dst = (T *)a.grad + row * a.grad_ld;
    // a scale of zero: padding, or nothing to learn from; zeros, whatever the logits hold
    if (first) {
      if (sh.repeated) {
        qj = 0.0;
        for (int j = 0; j < a.top; ++j) if (sh.id[j] == t.id) qj += sh.q[j];
      }
      dst[t.id] = from_f<T>(scale == 0.f ? 0.f : (float)((double)scale * (tr.total * (double)ex2(fmaf(z - ref, ch, -d)) - qj)));
    }
    write_row<T>(sr, dst, scale == 0.f, [&](int k) { return vals[k * NT]; }, [&](int g) { return (uint32_t)flags[g]; }, sr.edge >= 0 && !listed_edge, le, ref, ch, d, coef);
  }
  if (rank == 0 && warp == NW - 1 && lane == 0) {
    double others = 0.0, tops = 0.0, qz = 0.0;
    if (a.cluster > 1) join_parts(others, tops, qz);
    else { join(others, tops); qz = sh.qz_row; }
    const double total = others + tops, lse = (double)rm * a.inv_tau + log(total);
    const bool none = total == 0.0;                         // no finite logit
    double loss = sh.entropy - qz * a.inv_tau + ((double)sh.total - (double)sh.rest) * lse;
    if (tail) {
      const double log_rest = others > 0.0 ? -log1p(tops / others) : others == 0.0 ? -INFINITY : others;
      if (sh.rest > 0.f) loss -= (double)sh.rest * log_rest;
      a.log_rest[row] = none ? -INFINITY : (float)log_rest;
    }
    a.loss[row] = (float)(sh.total == 0.f ? 0.0 : none ? (double)INFINITY : loss);
    a.lse[row] = none ? -INFINITY : (float)lse;
  }
}

// The gradient from a saved log-sum-exp (and, with teacher_lse, log_rest).  A CTA walks `cta_vecs` vectors of a row with a ring of copies ahead
// of it.
template <typename T>
__global__ void __launch_bounds__(DISTILL_THREADS)
k_distill_grad(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  __shared__ TeacherSums teacher;
  __shared__ double sq[DISTILL_MAX_TOP];
  __shared__ int sid[DISTILL_MAX_TOP];
  constexpr int VEC = 16 / sizeof(T), NT = DISTILL_THREADS;
  kernel_entry(TR_k_distill_grad);
  const int row = blockIdx.x / a.cluster, tid = threadIdx.x;
  const RowShare<T> sr(a.logits, a.ld, row, a.vocab, blockIdx.x - row * a.cluster, a.cluster, a.cta_vecs);
  uint4 *vals = reinterpret_cast<uint4 *>(smem_raw) + tid;
  T *dst = (T *)a.grad + row * a.grad_ld;
  const float rs = a.row_scale ? a.row_scale[row] : 1.f;
  auto none = [](int) { return make_uint4(0u, 0u, 0u, 0u); };
  auto nobody = [](int) { return 0u; };
  if (rs == 0.f || a.lse[row] == -INFINITY) {               // a row of padding is not read
    write_row<T>(sr, dst, true, none, nobody, sr.edge >= 0, 0.f, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  auto fetch = [&](int k) {
    if (k * NT + tid < sr.nv) cp_async16(vals + k % DISTILL_GRAD_RING * NT, sr.mine + (size_t)k * NT * VEC);
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < DISTILL_GRAD_RING; ++k) fetch(k);
  const float le = sr.edge >= 0 ? to_f(sr.row[sr.edge]) : -INFINITY;
  const double lse = (double)a.lse[row];
  Entry t = {-1, -INFINITY, 0.0};
  if (tid >> 5 < teacher_warps(a)) {
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
  const bool mine = sr.flag_bit(t.id, a.vocab, blockIdx.x - row * a.cluster, a.cluster) >= 0 && scale != 0.0;
  float g_top = 0.f;
  if (tid < DISTILL_MAX_TOP) { sq[tid] = t.e * tr.mine(); sid[tid] = t.id; }
  __syncthreads();
  if (mine) {                                               // every entry of an id computes the same value
    double qj = 0.0;
    for (int j = 0; j < a.top; ++j) if (sid[j] == t.id) qj += sq[j];
    g_top = (float)(scale * (tr.total * exp((double)to_f(sr.row[t.id]) * a.inv_tau - lse) - qj));
  }
  __syncthreads();                                          // before any gradient is written: the two may be one buffer
  write_row<T>(sr, dst, scale == 0.0, [&](int k) {
    cp_async_wait<DISTILL_GRAD_RING - 1>();
    const uint4 q = vals[k % DISTILL_GRAD_RING * NT];
    fetch(k + DISTILL_GRAD_RING);
    return q;
  }, nobody, sr.edge >= 0, le, ref, ch, d, coef);
  cp_async_wait<0>();
  __syncthreads();
  if (mine) dst[t.id] = from_f<T>(g_top);
}
