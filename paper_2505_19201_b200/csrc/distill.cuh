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
// ids and of the row are in double.  At 6.45 TB/s of a copy:
//   4096 rows of 32000 bf16, 16 listed, with gradient: 116 us, 4.5 TB/s; 1024 rows of 262144 bf16: 270 us, 4.0 TB/s, fp32: 594 us, 3.6 TB/s
//   loss alone, 1000 rows of 131072 fp32: 102 us, 5.1 TB/s; 256 rows of 32000 bf16: 10.1 us, a launch and a row's chain of steps
//   gradient alone, 2048 rows of 32000 bf16, a fifth of them padding: 45 us, 5.4 TB/s; 777 rows of 49155 fp32: 60 us, 5.1 TB/s
// Between 4.5 and 6.45 TB/s stand the turnaround from a row's sums to its gradient and the exponentials (45 % of their units' rate).
#pragma once
#include "common.cuh"

#define DISTILL_MAX_TOP 128
#define DISTILL_THREADS 256
#define DISTILL_MAX_CLUSTER 8
#define DISTILL_MAX_VOCAB 262144

struct DistillArgs {
  const void *logits;
  long long ld;
  int rows, vocab, cluster, cta_vecs, top, alike;      // alike: all rows lie alike on 16-byte boundaries
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
// The largest of a warp's floats, NaN passed over.
__device__ __forceinline__ float max_of_warp(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
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
  float m, top_m;                      // largest logit that is not listed, that is; -inf without one
  double others, tops, qz;             // sums relative to these; sum of q_j z_j tau
};
// What the side warp knows of a row before its sums.
struct DistillSide {
  float total, rest, top_m;            // Q; q_r; largest listed logit of this share
  double tops;                         // the listed ids' sum relative to it, in double: see sums()
  double qz, entropy;                  // sum of q_j z_j tau in this share; sum of q ln q, the bucket's too
  double listed, left;                 // sum of q_j, and q_r: in the loss they multiply logarithms that all but cancel
};
template <int SW> struct DistillShared {
  DistillPart part[2][DISTILL_MAX_CLUSTER];
  DistillSide side[4];
  float2 pair[2][SW];                  // (maximum, sum) of every stream warp
  float q[DISTILL_MAX_TOP];            // for ids that are listed twice
  int id[DISTILL_MAX_TOP];
};
// Shared memory behind it, twice: a byte per vector of the CTA's share, whose bits say which ids are listed, and 16 bytes of such bits for the
// ids at the row's ends.  Then the ring of vectors.
#define DISTILL_PER 16                 // vectors of a thread in a block of the share
__host__ __device__ inline int distill_flag_bytes(int cta_vecs, int threads) {
  return (cta_vecs + DISTILL_PER * threads - 1) / (DISTILL_PER * threads) * (DISTILL_PER * threads) + 16;
}

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
  __device__ __forceinline__ RowShare(const void *p, long long ld, int r, int vocab, int rank, int cluster, int cta_vecs, int tid) {
    row = (const T *)p + r * ld;
    const int head = min(vocab, (VEC - (int)((uintptr_t)row / sizeof(T) % VEC)) % VEC), all = (vocab - head) / VEC,
              rest = vocab - head - all * VEC, v0 = min(all, rank * cta_vecs);
    id0 = head + v0 * VEC;
    nv = min(cta_vecs, all - v0);
    mine = row + id0 + tid * VEC;
    edge = rank == 0 && tid < head ? tid : rank == cluster - 1 && tid >= 16 && tid < 16 + rest ? vocab - rest + tid - 16 : -1;
  }
  // Where a listed id is in the share: a bit of its vector's byte, a thread's DISTILL_PER vectors of a block side by side, or of the bytes of the
  // edges from byte `edges` on; -1 elsewhere.
  template <int NT> __device__ __forceinline__ int flag_bit(int id, int rank, int cluster, int edges) const {
    const int at = id - id0;
    if (id < 0) return -1;
    if (at >= 0 && at < nv * VEC) {
      const int v = at / VEC, in = v % (DISTILL_PER * NT);
      return (((v / (DISTILL_PER * NT) * NT + in % NT) * DISTILL_PER + in / NT) << 3) + at % VEC;
    }
    if (at < 0) return rank == 0 && id0 < VEC ? edges * 8 + id : -1;                  // in front of the first boundary
    return rank == cluster - 1 ? edges * 8 + 16 + at - nv * VEC : -1;                 // behind the last
  }
};

// A vector of a gradient; vec: it lies on a 16-byte boundary.
template <typename T> __device__ __forceinline__ void store_vec(T *p, bool vec, const uint4 &q) {
  if (vec) { *reinterpret_cast<uint4 *>(p) = q; return; }
  constexpr int VEC = 16 / sizeof(T);
  T t[VEC];
  memcpy(t, &q, 16);
#pragma unroll
  for (int e = 0; e < VEC; ++e) p[e] = t[e];
}
// The gradient coef * 2^((l - ref) log2(e) / tau - d) of the thread's vectors, get(k) being the k-th's logits, and of its single id's logit le.
// Nothing is got where it is zero.  In fp32 the factor is two floats: what one is off by, 3e-8 of an exponent of 13, is the same for most of
// a row of 8192.  The first is rounded down, so that both are above 0 and a logit of -inf gives -inf.
template <typename T, typename F>
__device__ __forceinline__ void write_row(const RowShare<T> &sr, T *dst, bool zero, F get, float le, float ref, double factor, float d, float coef) {
  constexpr int VEC = 16 / sizeof(T), NT = DISTILL_THREADS;
  constexpr bool FULL = sizeof(T) == 4;
  const float ch = FULL ? __double2float_rz(factor * (1.0 - 0x1p-25)) : (float)factor, cl = (float)(factor - (double)ch);
  const float2 r2 = make_float2(-ref, -ref), c2 = make_float2(ch, ch), cl2 = make_float2(cl, cl), d2 = make_float2(-d, -d),
               o2 = make_float2(coef, coef);
  T *p = dst + sr.id0 + threadIdx.x * VEC;
  const bool vec = ((uintptr_t)p & 15) == 0;
  if (sr.edge >= 0) dst[sr.edge] = from_f<T>(zero ? 0.f : coef * ex2(fmaf(le - ref, ch, FULL ? fmaf(le - ref, cl, -d) : -d)));
  for (int k = 0, g = threadIdx.x; g < sr.nv; ++k, g += NT, p += NT * VEC) {
    uint4 q = make_uint4(0u, 0u, 0u, 0u);
    if (!zero) {
      float l[VEC];
      unpack_vec<T, VEC>(get(k), l);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 x = add_pair(make_float2(l[e], l[e + 1]), r2), y = fma_pair(x, c2, FULL ? fma_pair(x, cl2, d2) : d2);
        const float2 o = mul_pair(make_float2(ex2(y.x), ex2(y.y)), o2);
        l[e] = o.x; l[e + 1] = o.y;
      }
      q = pack_vec<T, VEC>(l);
    }
    store_vec<T>(p, vec, q);
  }
}

// Rows in a loop: cluster c takes the rows c, c + clusters, ..  SW stream warps walk a row's vectors, once for its sums and, with GRAD, once
// more for its gradient; one side warp does meanwhile what is left: the listed ids of the next row and the loss of the last.
// A stream thread has the same vectors in both passes, so its copies into shared memory need no barrier.  It walks blocks of 16 vectors of its own
// (with GRAD a share is one block), and a vector's place is taken by the next block's, or the next row's, as soon as its gradient is
// out (without GRAD: as soon as it has been added), so loads are always on their way.  (With a block per row and its own 64 KB the turnaround
// of the blocks cost as much as everything else: 4096 rows of 32000 bf16 with gradient took 152 us, 99 of them with both passes left out.)
// The side warp is the block's first: of the warps that could go on the oldest does, and as the last one it got a turn every 30 cycles and held
// the others up (127 us instead of 117).
#define DISTILL_GRAD_RING 8
#define DISTILL_SAVED_MAX 16777216.f
template <int THREADS> __device__ __forceinline__ void block_barrier() { asm volatile("barrier.sync 0, %0;" ::"n"(THREADS) : "memory"); }

template <typename T, bool GRAD, int SW>
struct DistillBlock {
  static constexpr int VEC = 16 / sizeof(T), NT = SW * 32, THREADS = NT + 32, PER = DISTILL_PER,
                       B = 4, TURNS = PER / B;       // vectors of a thread per turn, turns of a block
  const DistillArgs &a;
  DistillShared<SW> &sh;
  uint8_t *flags;                      // [2][distill_flag_bytes(cta_vecs)]
  int rank, first_row, clusters;
  // log2(e) / tau as a float, and 1 / tau as that float has it: the student's temperature in all of a row, off by up to 6e-8.  With q being
  // exact that changes the loss by 6e-8 of sum (q - p) z / tau; were tau itself taken in parts of it, by 6e-8 of sum p z / tau.
  float ch;
  double inv_tau;
  __device__ __forceinline__ uint8_t *flags_of(int p) const { return flags + p * distill_flag_bytes(a.cta_vecs, NT); }
  __device__ __forceinline__ RowShare<T> share(int row) const { return RowShare<T>(a.logits, a.ld, row, a.vocab, rank, a.cluster, a.cta_vecs, (int)threadIdx.x - 32); }
  __device__ __forceinline__ int edge_byte() const { return distill_flag_bytes(a.cta_vecs, NT) - 16; }
  // The sums of row i of the block, by a whole warp: of the others relative to their largest logit m, with the bucket of the listed ids relative
  // to theirs (without it the listed ids are among the others, and tops is 0).  Each keeps its own reference: between the two may lie more
  // than a float's range, at a low temperature in any row.
  // The exponentials of the others are all off in one direction by some 1e-7.  Where the listed ids' sum is exact, such an error e changes
  // the loss by e times the difference of the teacher's and the student's share of the listed ids; with the same error there it would change
  // it by e times the share itself, which in rows that nearly agree is much of the loss.  So the listed ids are summed by exp in double.
  // Every group of G lanes holds the G values, so that log2(G) exchanges add them up.
  template <typename R> struct Sums {
    float m, top_m;
    R others, tops;
    double qz;                           // where R is double
  };
  __device__ __forceinline__ void own_pairs(int i, float &m, double &others) const {
    const int lane = threadIdx.x & 31;
    const float2 p = sh.pair[i & 1][lane % SW];
    m = max_of_warp(p.x);
    others = group_sum<SW>((double)(p.x > -INFINITY ? p.y * ex2((p.x - m) * ch) : p.y));
  }
  template <int G, typename R> static __device__ __forceinline__ R group_sum(R v) {
#pragma unroll
    for (int x = G / 2; x > 0; x >>= 1) v += __shfl_xor_sync(0xffffffffu, v, x);
    return v;
  }
  template <typename R> __device__ __forceinline__ Sums<R> sums(int i) const {
    const int lane = threadIdx.x & 31;
    const bool tail = a.teacher_lse != nullptr;
    Sums<R> r;
    r.top_m = -INFINITY; r.tops = 0;
    if (a.cluster == 1) {
      const float2 p = sh.pair[i & 1][lane % SW];
      if (tail) { r.top_m = sh.side[i & 3].top_m; r.tops = (R)sh.side[i & 3].tops; }
      r.qz = sh.side[i & 3].qz;
      r.m = max_of_warp(p.x);
      r.others = group_sum<SW>((R)(p.x > -INFINITY ? p.y * ex2((p.x - r.m) * ch) : p.y));
    } else {
      constexpr int G = DISTILL_MAX_CLUSTER;
      const bool on = lane % G < a.cluster;
      const DistillPart &x = sh.part[i & 1][lane % G];
      const float m = on ? x.m : -INFINITY;
      r.m = max_of_warp(m);
      R o = on ? (R)x.others : (R)0;
      if (m > -INFINITY) o *= ex2((m - r.m) * ch);
      r.others = group_sum<G>(o);
      if (tail) {
        const float tm = on ? x.top_m : -INFINITY;
        r.top_m = max_of_warp(tm);
        R t = on ? (R)x.tops : (R)0;
        if (tm > -INFINITY) {
          if constexpr (sizeof(R) == 8) t *= exp(((double)tm - (double)r.top_m) * inv_tau);
          else t *= ex2((tm - r.top_m) * ch);
        }
        r.tops = group_sum<G>(t);
      }
      if constexpr (sizeof(R) == 8) r.qz = group_sum<G>(on ? x.qz : 0.0);
    }
    return r;
  }
  // The gradient of an id that is not listed is coef * 2^((l - ref) ch), ref the largest of their logits.
  struct Slope { float ref, scale, coef; };
  __device__ __forceinline__ Slope slope(int i, float rs) const {
    Slope g;
    const Sums<float> s = sums<float>(i);
    const float q = sh.side[i & 3].total;
    float total = s.others, part = q;                       // Q - q_r / p_r, times p_r
    if (a.teacher_lse) {                                    // p_r Q - q_r, without the p_r q_r that both have
      const float rm = fmaxf(s.m, s.top_m), o = s.m > -INFINITY ? s.others * ex2((s.m - rm) * ch) : s.others,
                  t = s.top_m > -INFINITY ? s.tops * ex2((s.top_m - rm) * ch) : s.tops;
      total = o + t;
      part = __fdividef((float)sh.side[i & 3].listed * o - sh.side[i & 3].rest * t, total);
    }
    g.ref = s.m > -INFINITY ? s.m : 0.f;
    g.scale = total == 0.f || q == 0.f ? 0.f : rs * (float)a.inv_tau;         // 0: padding, or nothing to learn from
    g.coef = g.scale == 0.f || s.others == 0.f ? 0.f : g.scale * __fdividef(part, s.others);
    return g;
  }

  // ---- the side warp: lane's entries are lane, lane + 32, ..
  static constexpr int E = DISTILL_MAX_TOP / 32;
  struct Entries { int id[E], bit[E]; float q[E]; bool first[E]; double w[E]; };      // bit: its mark's place, -1 outside the share; w: e^(z / tau)
                                                                                      // relative to the largest listed logit of the share
  __device__ __forceinline__ void load_entries(int row, int (&id)[E], float (&t)[E]) const {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = lane + 32 * i;
      id[i] = -1; t[i] = -INFINITY;
      if (j < a.top && row < a.rows) {
        id[i] = a.ids[(long long)row * a.top + j];
        t[i] = a.teacher[(long long)row * a.top + j];
        if (id[i] < 0 || id[i] >= a.vocab) id[i] = -1;
      }
    }
  }
  // Marks the listed ids of a row, the i-th of the block, whose entries are id and t, and leaves sh.side[i & 3].
  __device__ __forceinline__ void prepare(int row, int i_row, const int (&id)[E], const float (&t)[E], Entries &n) const {
#pragma unroll
    for (int i = 0; i < E; ++i) { n.id[i] = id[i]; n.bit[i] = -1; n.first[i] = false; n.w[i] = 0.0; n.q[i] = 0.f; }
    if (row >= a.rows) return;
    const int lane = threadIdx.x & 31;
    const RowShare<T> sr = share(row);
    uint32_t *words = reinterpret_cast<uint32_t *>(flags_of(i_row & 1));
    double x[E], e[E], ref = -INFINITY, s = 0.0, l = 0.0, qz = 0.0;
    float z[E], tm = -INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = -INFINITY; z[i] = -INFINITY;
      if (i * 32 >= a.top) continue;
      n.bit[i] = sr.template flag_bit<NT>(n.id[i], rank, a.cluster, edge_byte());
      if (n.bit[i] >= 0) z[i] = to_f(sr.row[n.id[i]]);
      n.first[i] = n.bit[i] >= 0;
      x[i] = n.id[i] >= 0 ? (double)t[i] * a.inv_tau : -INFINITY;
      sh.id[lane + 32 * i] = n.id[i];
    }
    bool twice = false;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (n.bit[i] >= 0 && (atomicOr(words + (n.bit[i] >> 5), 1u << (n.bit[i] & 31)) >> (n.bit[i] & 31) & 1u)) twice = true;
    twice = __any_sync(0xffffffffu, twice);
    __syncwarp();
    if (twice) {                                            // of the entries of one id the first stands for it
#pragma unroll
      for (int i = 0; i < E; ++i)
        for (int j = 0; j < lane + 32 * i; ++j) if (sh.id[j] == n.id[i]) n.first[i] = false;
    }
    if (a.teacher_lse) ref = (double)a.teacher_lse[row];
    else {
#pragma unroll
      for (int i = 0; i < E; ++i) ref = fmax(ref, x[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ref = fmax(ref, __shfl_xor_sync(0xffffffffu, ref, o));
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      e[i] = 0.0;
      if (i * 32 < a.top) {
        if (n.id[i] >= 0 && x[i] != -INFINITY) e[i] = exp(x[i] - ref);
        s += e[i];
        if (!(e[i] == 0.0)) {
          l += e[i] * (a.teacher_lse ? x[i] - ref : x[i]);
          if (n.bit[i] >= 0) qz += e[i] * (double)z[i];
        }
        tm = fmaxf(tm, z[i]);
      }
    }
    tm = max_of_warp(tm);
    double ts = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (i * 32 < a.top && (GRAD || a.teacher_lse)) {
        if (n.first[i] && z[i] != -INFINITY) n.w[i] = exp(((double)z[i] - (double)tm) * inv_tau);
        ts += n.w[i];
      }
    ts = warp_sum_d(ts); s = warp_sum_d(s); l = warp_sum_d(l); qz = warp_sum_d(qz);
    const bool any = !(s == 0.0);                           // a row with no valid entry has no loss, with or without the rest
    DistillSide d;
    double f = 1.0, rest = 0.0;
    if (a.teacher_lse) {
      rest = any ? fmax(0.0, 1.0 - s) : 0.0;
      d.total = any ? (float)(s + rest) : 0.f;
      d.entropy = l + (rest > 0.0 ? rest * log(rest) : 0.0);
    } else {
      f = any ? 1.0 / s : 0.0;
      d.total = any ? 1.f : 0.f;
      d.entropy = any ? l * f - (ref + log(s)) : 0.0;
    }
    d.rest = (float)rest;
    d.left = rest;
    d.listed = any ? s * f : 0.0;
    d.qz = qz == 0.0 ? 0.0 : qz * f;
    d.top_m = tm; d.tops = ts;
#pragma unroll
    for (int i = 0; i < E; ++i) n.q[i] = (float)(e[i] * f);     // in single precision: doubles for two rows spill (8 % of a step)
    if (twice) {
#pragma unroll
      for (int i = 0; i < E; ++i) sh.q[lane + 32 * i] = n.q[i];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (n.first[i]) {
          n.q[i] = 0.f;
          for (int j = 0; j < a.top; ++j) if (sh.id[j] == n.id[i]) n.q[i] += sh.q[j];
        }
      __syncwarp();
    }
    if (lane == 0) sh.side[i_row & 3] = d;
    __syncwarp();
  }
  // The row's results; returns what turns the weights of the listed ids of this share into Q p.  The few functions in double are of this warp's
  // time between two rows' barriers, and a chain of them one by one (two logarithms, a quotient and five exponentials) was a tenth of all, so
  // the lanes take each an argument of their own.
  __device__ __forceinline__ double finish(int row, int i, bool &none) const {
    const int lane = threadIdx.x & 31;
    Sums<double> s = sums<double>(i);
    const DistillSide &d = sh.side[i & 3];
    // ex2.approx is 5.1e-8 below 2^x in the mean, measured over -28 < x < 0; the largest logit's own term is 1 and exact
    s.others += 5.1e-8 * fmax(s.others - 1.0, 0.0);
    const float rm = fmaxf(s.m, s.top_m);
    double total = s.others, log_total = 0.0, p_r = 0.0, log_rest = 0.0, own = 0.0;
    if (a.teacher_lse) {
      // relative to rm: 0 the others, 1 the listed ids, 4 those of this share; the listed to the others: 2, 3
      const double from = (double)(lane == 0 ? s.m : lane == 4 ? d.top_m : s.top_m), to = (double)(lane == 2 || lane == 3 ? s.m : rm),
                   gap = (from - to) * (lane == 3 ? a.inv_tau : inv_tau), e = exp(fmin(gap, 600.0));
      total = s.others * __shfl_sync(0xffffffffu, e, 0) + s.tops * __shfl_sync(0xffffffffu, e, 1);
      own = __shfl_sync(0xffffffffu, e, 4);
      // ln total, and ln (1 + listed / others) = -ln p_r
      if (rank == 0) {
        const double lg = log1p(lane < 2 ? total - 1.0 : s.tops / s.others * e) + (lane >= 2 && gap > 600.0 ? gap - 600.0 : 0.0);
        log_total = __shfl_sync(0xffffffffu, lg, 0); p_r = __shfl_sync(0xffffffffu, lg, 2); log_rest = __shfl_sync(0xffffffffu, lg, 3);
      }
    } else {
      if (rank == 0) log_total = log(total);
      if (GRAD) own = exp(((double)d.top_m - (double)rm) * inv_tau);
    }
    none = total == 0.0;                                    // no finite logit
    if (rank == 0) {
      const double no_rest = s.others == 0.0 ? INFINITY : s.others;         // or NaN
      double loss = d.entropy - s.qz * inv_tau + d.listed * ((double)rm * inv_tau + log_total);
      if (d.left > 0.0) loss += d.left * (s.others > 0.0 ? p_r : no_rest);
      if (lane == 0) {
        if (a.teacher_lse) a.log_rest[row] = none ? -INFINITY : (float)-(s.others > 0.0 ? log_rest : no_rest);
        a.loss[row] = (float)(d.total == 0.f ? 0.0 : none ? (double)INFINITY : loss);
        a.lse[row] = none ? -INFINITY : (float)((double)rm * a.inv_tau + log_total);
      }
    }
    return none ? 0.0 : own * (double)d.total / total;
  }
  // One barrier to a row, when its sums are there.  Behind it the stream warps write the row's gradient and go on to the next row, while this warp
  // replaces the gradients of the listed ids of the row before, whose others are all out by now, computes this row's, finishes its loss and
  // prepares the row after the next, whose marks take the place of this row's.
  __device__ __forceinline__ void side_warp() const {
    Entries n, next;
    int id[E];
    float t[E], g_top[E];
    load_entries(first_row, id, t);
    for (int i = threadIdx.x & 31; i < distill_flag_bytes(a.cta_vecs, NT) * 2 / 4; i += 32) reinterpret_cast<uint32_t *>(flags)[i] = 0;
    __syncwarp();
    prepare(first_row, 0, id, t, n);
    load_entries(first_row + clusters, id, t);
    prepare(first_row + clusters, 1, id, t, next);
    cluster_started_wait(a.cluster);
    block_barrier<THREADS>();
    int i_row = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) { g_top[i] = 0.f; id[i] = -1; }             // id: of the row before, where this warp has something to write
#pragma unroll 1
    for (int row = first_row; row < a.rows; row += clusters, ++i_row) {
      const float rs = GRAD && a.row_scale ? a.row_scale[row] : 1.f;
      block_barrier<THREADS>();
      if (a.cluster > 1) {
        const int lane = threadIdx.x & 31;
        float m;
        double others;
        own_pairs(i_row, m, others);
        if (lane < a.cluster) {
          const uint32_t to = mapa(smem_u32(&sh.part[i_row & 1][rank]), lane);
          st_cluster_u64(to, (unsigned long long)__float_as_uint(m) | (unsigned long long)__float_as_uint(sh.side[i_row & 3].top_m) << 32);
          st_cluster_u64(to + 8, __double_as_longlong(others));
          st_cluster_u64(to + 16, __double_as_longlong(sh.side[i_row & 3].tops));
          st_cluster_u64(to + 24, __double_as_longlong(sh.side[i_row & 3].qz));
        }
        cluster_sync_all();
      }
      int ahead[E];
      load_entries(row + 2 * clusters, ahead, t);
      if (GRAD && i_row) write_listed(row - clusters, id, g_top);
      double p = 0.0;
      bool none = false;
      if (GRAD || rank == 0) p = finish(row, i_row, none);
      if (GRAD) {
        const double scale = none || sh.side[i_row & 3].total == 0.f ? 0.0 : (double)rs * a.inv_tau;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          id[i] = n.first[i] ? n.id[i] : -1;
          g_top[i] = scale == 0.0 ? 0.f : (float)(scale * (p * n.w[i] - (double)n.q[i]));
        }
      }
#pragma unroll
      for (int i = 0; i < E; ++i) if (i * 32 < a.top && n.bit[i] >= 0) flags_of(i_row & 1)[n.bit[i] >> 3] = 0;
      __syncwarp();
      n = next;
      prepare(row + 2 * clusters, i_row + 2, ahead, t, next);
    }
    block_barrier<THREADS>();
    if (GRAD) write_listed(first_row + (i_row - 1) * clusters, id, g_top);
  }
  __device__ __forceinline__ void write_listed(int row, const int (&id)[E], const float (&g_top)[E]) const {
    T *dst = (T *)a.grad + row * a.grad_ld;
#pragma unroll
    for (int i = 0; i < E; ++i) if (id[i] >= 0) dst[id[i]] = from_f<T>(g_top[i]);
  }

  // ---- the stream warps
  // The vectors of a turn of the next block, where the block has them (left: ids of vectors from the thread's first on), as one group of copies.
  // The passes are loops over turns whose body is as short as it gets: unrolled over a block they waited for instructions more than
  // for anything else.
  __device__ __forceinline__ void fetch(int turn, const T *from, int left, uint4 *ring) const {
#pragma unroll
    for (int k = 0; k < B; ++k)
      if ((turn * B + k) * NT < left) cp_async16(ring + (turn * B + k) * NT, from + (turn * B + k) * NT * VEC);
    cp_async_commit();
  }
  // A turn's vectors; without one -inf.  ring and left are the turn's own.
  __device__ __forceinline__ void take(const uint4 *ring, int left, uint4 (&q)[B]) const {
    if ((B - 1) * NT < left) {
#pragma unroll
      for (int k = 0; k < B; ++k) q[k] = ring[k * NT];
    } else {
      const uint32_t u = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
#pragma unroll
      for (int k = 0; k < B; ++k) q[k] = k * NT < left ? ring[k * NT] : make_uint4(u, u, u, u);
    }
  }
  __device__ __forceinline__ void add_turn(const uint4 *ring, int left, uint32_t listed, float &m, float &ref, float2 &s) const {
    uint4 q[B];
    take(ring, left, q);
    if (listed) {
#pragma unroll
      for (int k = 0; k < B; ++k) {
        T t[VEC];
        memcpy(t, &q[k], 16);
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (listed >> (k * 8 + e) & 1u) t[e] = from_f<T>(-INFINITY);
        memcpy(&q[k], t, 16);
      }
    }
    float v = max_vec<T, VEC>(q[0]);
#pragma unroll
    for (int k = 1; k < B; ++k) v = fmaxf(v, max_vec<T, VEC>(q[k]));
    if (v > m) {
      if (m > -INFINITY) { const float f = ex2((m - v) * ch); s.x *= f; s.y *= f; }
      m = ref = v;
    }
    const float2 r2 = make_float2(-ref, -ref), c2 = make_float2(ch, ch);
#pragma unroll
    for (int k = 0; k < B; ++k) {
      float l[VEC];
      unpack_vec<T, VEC>(q[k], l);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = mul_pair(add_pair(make_float2(l[e], l[e + 1]), r2), c2);
        s = add_pair(s, make_float2(ex2(y.x), ex2(y.y)));
      }
    }
  }
  __device__ __forceinline__ void write_turn(const uint4 *ring, int left, T *out, bool vec, const Slope &g) const {
    const float2 r2 = make_float2(-g.ref, -g.ref), c2 = make_float2(ch, ch), o2 = make_float2(g.coef, g.coef);
    uint4 q[B];
    take(ring, left, q);
#pragma unroll
    for (int k = 0; k < B; ++k) {
      float l[VEC];
      unpack_vec<T, VEC>(q[k], l);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 y = mul_pair(add_pair(make_float2(l[e], l[e + 1]), r2), c2);
        const float2 o = mul_pair(make_float2(ex2(y.x), ex2(y.y)), o2);
        l[e] = o.x; l[e + 1] = o.y;
      }
      if (k * NT < left) store_vec<T>(out + k * NT * VEC, vec, pack_vec<T, VEC>(l));
    }
  }
  __device__ __forceinline__ void stream_warp(uint4 *ring) const {
    const int tid = (int)threadIdx.x - 32, lane = tid & 31, warp = tid >> 5;
    const bool tail = a.teacher_lse != nullptr;
    RowShare<T> sr = share(first_row), next = sr;
#pragma unroll
    for (int t = 0; t < TURNS; ++t) fetch(t, sr.mine, sr.nv - tid, ring);
    float le = sr.edge >= 0 ? to_f(sr.row[sr.edge]) : -INFINITY;
    cluster_started_wait(a.cluster);
    block_barrier<THREADS>();
    int i_row = 0;
#pragma unroll 1
    for (int row = first_row; row < a.rows; row += clusters, ++i_row) {
      const uint8_t *fl = flags_of(i_row & 1);
      const bool more = row + clusters < a.rows;
      if (more) {
        if (a.alike) { next.row += clusters * a.ld; next.mine += clusters * a.ld; }
        else next = share(row + clusters);
      }
      // running maximum m (ref: the same, 0 without one) and sum of 2^((l - ref) ch); listed ids stay out where the rest is a bucket
      float m = -INFINITY, ref = 0.f;
      float2 s = make_float2(0.f, 0.f);
      if (sr.edge >= 0 && !(tail && (fl[edge_byte() + (tid >> 3)] >> (tid & 7) & 1u))) {
        if (le > m) { m = ref = le; s.x = 1.f; }
        else if (le != le) s.x = le;
      }
      const float rs = GRAD && a.row_scale ? a.row_scale[row] : 1.f;
      const T *from = sr.mine;
      int left = sr.nv - tid, block = 0;
#pragma unroll 1
      do {
        const uint8_t *marks = fl + (block * NT + tid) * PER;
        const bool last = GRAD || sr.nv <= (block + 1) * PER * NT;
        from = last ? next.mine : from + PER * NT * VEC;
        const int from_left = last ? (more ? next.nv - tid : 0) : left - PER * NT;
#pragma unroll 1
        for (int t = 0; t < TURNS; ++t) {
          if (!GRAD) cp_async_wait<TURNS - 1>();
          else if (t == 0) cp_async_wait<TURNS / 2>();
          else if (t == TURNS / 2) cp_async_wait<0>();
          const int here = left - t * B * NT;
          if (here > 0) add_turn(ring + t * B * NT, here, tail ? *reinterpret_cast<const uint32_t *>(marks + t * B) : 0u, m, ref, s);
          if (!GRAD) fetch(t, from, from_left, ring);
        }
        left -= PER * NT;
        ++block;
      } while (!GRAD && sr.nv > block * PER * NT);
      const float wm = max_of_warp(m);
      s.x = warp_sum((s.x + s.y) * (m > -INFINITY ? ex2((m - wm) * ch) : 1.f));       // without a maximum 0, or NaN
      if (lane == 0) sh.pair[i_row & 1][warp] = make_float2(wm, s.x);
      block_barrier<THREADS>();
      if (a.cluster > 1) cluster_sync_all();
      const float le_now = le;
      if (more) le = next.edge >= 0 ? to_f(next.row[next.edge]) : -INFINITY;
      if (GRAD) {
        const Slope g = slope(i_row, rs);
        T *dst = (T *)a.grad + row * a.grad_ld, *out = dst + sr.id0 + tid * VEC;
        const bool vec = ((uintptr_t)out & 15) == 0;
        const int from_left = more ? next.nv - tid : 0;
        left = sr.nv - tid;
        if (sr.edge >= 0) dst[sr.edge] = from_f<T>(g.scale == 0.f ? 0.f : g.coef * ex2((le_now - g.ref) * ch));
#pragma unroll 1
        for (int t = 0; t < TURNS; ++t) {
          const int here = left - t * B * NT;
          if (here > 0) {
            if (g.scale != 0.f) write_turn(ring + t * B * NT, here, out + t * B * NT * VEC, vec, g);
            else                                            // zeros, whatever the logits hold
              for (int k = 0; k < B; ++k)
                if (k * NT < here) store_vec<T>(out + (t * B + k) * NT * VEC, vec, make_uint4(0u, 0u, 0u, 0u));
          }
          fetch(t, next.mine, from_left, ring);
        }
      }
      sr = next;
    }
    block_barrier<THREADS>();
    cp_async_wait<0>();
  }
};

// GRAD: the gradient leaves in the same call.
template <typename T, bool GRAD, int SW>
__global__ void __launch_bounds__((SW + 1) * 32, SW == 8 ? 3 : 1)
k_distill(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillShared<SW> &sh = *reinterpret_cast<DistillShared<SW> *>(smem_raw);
  uint8_t *flags = smem_raw + (sizeof(DistillShared<SW>) + 15) / 16 * 16;
  cluster_started_arrive(a.cluster);
  kernel_entry(TR_k_distill);
  const DistillBlock<T, GRAD, SW> blk = {a, sh, flags, a.cluster > 1 ? (int)cluster_ctarank() : 0, (int)blockIdx.x / a.cluster, (int)gridDim.x / a.cluster,
                                         (float)(a.inv_tau * 1.4426950408889634), (double)(float)(a.inv_tau * 1.4426950408889634) * 0.6931471805599453};
  if (threadIdx.x < 32) blk.side_warp();
  else blk.stream_warp(reinterpret_cast<uint4 *>(flags + 2 * distill_flag_bytes(a.cta_vecs, SW * 32)) + threadIdx.x - 32);
}

// The gradient from a saved log-sum-exp (and, with teacher_lse, log_rest).  Both are floats, whose rounding, 2^-25 to 2^-24 of their size, is the
// exponents' error.  Beyond 2^24 that is more than 1/2: a float of -1e9 is off by up to 32, and e^32 of a row that is masked with it would be its
// gradient.  (The call that makes both in one pass has the sums themselves.)  A CTA walks `cta_vecs` vectors of a row with a ring of copies ahead
// of it.
template <typename T>
__global__ void __launch_bounds__(DISTILL_THREADS, 5)
k_distill_grad(const __grid_constant__ DistillArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  __shared__ TeacherSums teacher;
  __shared__ double sq[DISTILL_MAX_TOP];
  __shared__ int sid[DISTILL_MAX_TOP];
  constexpr int VEC = 16 / sizeof(T), NT = DISTILL_THREADS;
  kernel_entry(TR_k_distill_grad);
  const int row = blockIdx.x / a.cluster, tid = threadIdx.x;
  const RowShare<T> sr(a.logits, a.ld, row, a.vocab, blockIdx.x - row * a.cluster, a.cluster, a.cta_vecs, tid);
  uint4 *vals = reinterpret_cast<uint4 *>(smem_raw) + tid;
  T *dst = (T *)a.grad + row * a.grad_ld;
  const float rs = a.row_scale ? a.row_scale[row] : 1.f;
  auto none = [](int) { return make_uint4(0u, 0u, 0u, 0u); };
  // A row of padding is not read; nor is one of which the saved lse says nothing (rows of nothing but logits masked with -1e9, say).
  if (rs == 0.f || fabsf(a.lse[row]) > DISTILL_SAVED_MAX) {
    write_row<T>(sr, dst, true, none, 0.f, 0.f, 0.0, 0.f, 0.f);
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
  // (p_r Q - q_r) times the id's part of the others, which is no more than 1 however small p_r is: logits relative to tau (lse + ln p_r)
  const bool rest = a.teacher_lse && !(a.log_rest[row] < -DISTILL_SAVED_MAX);
  const double rest_log = rest ? (double)a.log_rest[row] : 0.0, base = lse + rest_log;
  const float ref = (float)(base / a.inv_tau),
              d = (float)((base - (double)ref * a.inv_tau) * 1.4426950408889634),
              coef = (float)(scale * (!a.teacher_lse ? tr.total : !rest ? 0.0 : tr.total * exp(rest_log) - tr.rest));
  const bool mine = sr.template flag_bit<NT>(t.id, blockIdx.x - row * a.cluster, a.cluster, 0) >= 0 && scale != 0.0;
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
  }, le, ref, a.inv_tau * 1.4426950408889634, d, coef);
  cp_async_wait<0>();
  __syncthreads();
  if (mine) dst[t.id] = from_f<T>(g_top);
}
