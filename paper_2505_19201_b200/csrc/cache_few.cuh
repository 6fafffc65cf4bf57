// Attention over a paged cache for up to four query entries per item (a token of one sequence and its KV head's group, a listed row), on the tcgen05 tensor
// cores.  How the work is dealt out: cache_work.cuh.
//
// The keys stand on the matrix instruction's long side:  S^T = K Q^T  (keys x 16), O^T += V^T P^T  (head_dim x 16).  Then every lane of every softmax warp has a key, four
// entries each, and nothing is computed for rows that are not there.  Against the kernel with the entries on the long side (cache_attn.cuh), whose two softmax warps of sixteen rows
// have all there is to do: 64 sequences of 2000 tokens, 32 heads over 8 of 128 wide, 89 us and 92 to 108; 12 heads of 64, 70 and 102 to 108; one of 833 tokens, 32 heads of 128, 13.0 and
// 14.4.  At 256 wide neither is ahead (16 over 8: 171 and 170 to 175; of 1000 tokens, two rows each, 94 and 92), and the rule is the same for all widths.  A form for up to 16 entries lost to the other kernel: 28 over 4 heads of 128 65 us against 53, 32 over 2 43 against 33, 24 over 3 of 64 38 against 35.
//   S^T   tcgen05.mma 128 x 16 x 16 over head_dim, A = the unit's keys and B = Q, both K-major; fp32 in TMEM, a ring of four 16-column buffers
//   softmax   four warps, a key per thread: P = 2^(s - m) with a running reference m per entry, the same in all threads.  Whether some score has outgrown its reference
//         by more than a power of two is one barrier with a vote per unit; only then (in the first unit of a segment, and seldom later) the maxima are taken, across lanes and warps, and
//         O^T, 16 columns, takes the new reference.  A thread sums its own keys' weights (rounded as the product takes them, and unrounded for
//         the log-sum-exp); they meet at the segment's end.
//   O^T   tcgen05.mma 128 x 16 x 16 over the keys, A = V as stored (MN-major), B = P in shared memory (K-major); two accumulators, so that a segment starts while the
//         one before it is read out.  A lane is a channel: what it stores is contiguous across the warp.
// Units of 128 keys (head_dim 256: 64, whose other 64 rows of the instruction are whatever lies behind them in shared memory, and nobody reads what comes of it; the same for the
// channels past 63 at head_dim 64).  K, V and Q come by TMA.  Bound by HBM: 24 rows of 48 pages, 32 heads over 8 of
// 128 in fp16, 302 MB in 55 us; three units of K and V ahead of each other are what shared memory holds.
// Warps: 0 K and segments, 1 Q and S, 2 O, 3 V, 4..7 softmax and epilogue.
#pragma once
#include "attn_tc.cuh"
#include "cache_work.cuh"

#define CF_THREADS 256
#define CF_ENTRIES 4                     // entries of a tile at most
#define CF_N 16                          // the N of the instructions: no fewer
#define CF_S 4                           // buffers of S
#define CF_START 3                       // units that starting and ending an item is worth: 128 sequences of up to 1000 tokens, 32 heads of 64, with 1, 2, 3: 179, 154, 151 us

template <int HD> struct CfShape {
  static constexpr int BLK = HD == 256 ? 64 : 128;                     // keys of a unit
  static constexpr int KP = HD / 64, PK = BLK / 64;                    // 64-column panels of a row, 64-key panels of P
  static constexpr int STAGES = 3;                                     // units of K (and of V) in shared memory
  static constexpr int MT = HD == 256 ? 2 : 1;                         // tiles of 128 channels
  static constexpr int CTAS_PER_SM = HD == 64 ? 2 : 1;                 // what shared memory holds
  static constexpr int STAGE = BLK * HD * 2, PANEL = BLK * 128;
  static constexpr int Q_PANEL = CF_N * 128, Q_BYTES = KP * Q_PANEL, P_PANEL = CF_N * 128, P_BYTES = PK * P_PANEL;
  static constexpr int O_COLS = MT * CF_N;
  static constexpr int TMEM_COLS = 128;                                // 4 x 16 for S, 2 x 32 at most for O
  static constexpr size_t SMEM = 1024 + 2 * STAGES * STAGE + 2 * Q_BYTES + 2 * P_BYTES + 2048;
};

__device__ __forceinline__ bool cf_any(bool mine) {                    // ... of the four softmax warps
  uint32_t r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 128, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"((uint32_t)mine) : "memory");
  return r != 0;
}
// Four columns of a warp's 32 lanes, a lane to a thread.
__device__ __forceinline__ void cf_ld(uint32_t taddr, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void cf_st(uint32_t taddr, const uint32_t (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void cf_sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }

template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(CF_THREADS, (CfShape<HD>::CTAS_PER_SM))
k_cache_attn_few(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
                 const __grid_constant__ CacheAttnArgs a) {
  using Sh = CfShape<HD>;
  constexpr int STAGES = Sh::STAGES, KP = Sh::KP, BLK = Sh::BLK, NE = CF_ENTRIES;
  extern __shared__ uint8_t cf_smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)cf_smem_raw + 1023) & ~(uintptr_t)1023);
  // V in front of K in front of Q: what an instruction reads past its rows (see above) is there
  uint8_t *v_s = smem, *k_s = v_s + STAGES * Sh::STAGE, *q_s = k_s + STAGES * Sh::STAGE, *p_s = q_s + 2 * Sh::Q_BYTES;
  uint64_t *bars = (uint64_t *)(p_s + 2 * Sh::P_BYTES);
  uint64_t *k_full = bars, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES;
  uint64_t *s_full = v_empty + STAGES, *s_empty = s_full + CF_S, *p_full = s_empty + CF_S, *o_done = p_full + 2, *o_free = o_done + 2;
  uint64_t *q_full = o_free + 2, *q_empty = q_full + 2, *seg_full = q_empty + 2;
  uint4 *masks = (uint4 *)(((uintptr_t)(seg_full + CA_RING) + 15) & ~(uintptr_t)15);                         // [CA_RING] which keys of a unit there are
  CaSeg *segs = (CaSeg *)(masks + CA_RING);                                // [CA_RING]
  uint32_t *tmem_base_p = (uint32_t *)(segs + CA_RING);
  volatile int *abort_flag = (volatile int *)(tmem_base_p + 1);
  __shared__ CaPlanShared plan;
  __shared__ int sh_status[2];
  __shared__ float red[4][NE];                                           // maxima of the warps
  __shared__ float2 sums[4][NE];                                         // their sums of weights
  __shared__ int e_vis[2][NE], e_row[2][NE], e_nodes[2][NE];           // of a segment's entries: what they see, their row, and its tree's nodes
  __shared__ void *e_to[NE];                                               // at its end: where O goes, the factor, the reference
  __shared__ float e_inv[NE], refs[NE];
  static_assert(CA_RING > STAGES + CF_S + 1, "what the producer leaves is read until a unit's P is done");
  static_assert(sizeof(uint64_t) * (4 * STAGES + 2 * CF_S + 10 + CA_RING) + sizeof(uint4) * CA_RING + sizeof(CaSeg) * CA_RING + 8 <= 2048, "room for the barriers and rings");

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, cta = blockIdx.x;
  unsigned long long *tr = trace_open();
  if (warp == 0) {
    if (lane < STAGES) { mbar_init(k_full + lane, 1); mbar_init(k_empty + lane, 1); mbar_init(v_full + lane, 1); mbar_init(v_empty + lane, 1); }
    else if (lane >= 4 && lane < 4 + CF_S) { mbar_init(s_full + lane - 4, 1); mbar_init(s_empty + lane - 4, 4); }
    else if (lane >= 8 && lane < 10) {
      const int i = lane - 8;
      mbar_init(p_full + i, 4); mbar_init(o_done + i, 1); mbar_init(o_free + i, 4); mbar_init(q_full + i, 1); mbar_init(q_empty + i, 1);
    } else if (lane >= 16) mbar_init(seg_full + lane - 16, 1);
    if (lane == 12) { *abort_flag = 0; plan.partial = plan.longest = 0; sh_status[0] = sh_status[1] = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_p)), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Behind the launch of this call for full tiles there is nothing to wait for: that one has waited for all in front of it before it let this one start.  (64 readers of a
  // prefix of 32768 keys, 64 wide: 226 -> 218 us.  Were this launch let start when the other one has begun, so that its CTAs follow those that leave one by one, it would
  // be no faster, and questions on one image slower, 36.3 us in place of 35.2.)
  if (!a.early) pdl_wait();
  if (a.let) pdl_trigger();
  trace_stamp(tr, TR_k_cache_attn);
  int *status = a.status ? a.status : sh_status;
  CaWalk<BLK, CF_START, PAGES> w;
  w.plan(a, plan, status);
  const uint32_t tmem_base = *tmem_base_p, o_base = tmem_base + CF_S * CF_N;
  int gave_up = WAIT_none;
  // Units of segment number i, once the producer has left it; 0: there is none, or a wait ran out.
  auto segment = [&](int i, int where) {
    if (!mbar_wait_warp(seg_full + i % CA_RING, (uint32_t)(i / CA_RING) & 1u, abort_flag)) { gave_up = where; return 0; }
    return segs[i % CA_RING].n;
  };

  if (warp == 0) {
    gave_up = ca_produce<HD, STAGES, 0>(a, w, CaRing{k_full, k_empty, seg_full, k_s, masks, segs, &map_k, abort_flag, status}, lane);
  } else if (warp == 3) {
    gave_up = ca_produce<HD, STAGES, 1>(a, w, CaRing{v_full, v_empty, nullptr, v_s, nullptr, nullptr, &map_v, abort_flag, status}, lane);
  } else if (warp == 1) {
    // ------------------------------------------------------------------ queries, a segment ahead, and S^T = K Q^T
    constexpr uint32_t idesc = (1u << 4) | CaType<T>::IDESC | ((uint32_t)(CF_N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t qd = smem_desc(smem_u32(q_s)), kd = smem_desc(smem_u32(k_s));
    const uint64_t pol = policy_evict_normal();
    int st = 0, sb = 0;
    uint32_t ph = 0, sph = 1;
    auto fetch = [&](int seg) {                             // queries of a segment into the buffer that the one before last has left (false: a wait ran out)
      if (segment(seg, WAIT_cache_q) <= 0) return !gave_up;
      const int qb = seg & 1;
      if (!mbar_wait_warp(q_empty + qb, (uint32_t)(seg >> 1 & 1) ^ 1u, abort_flag)) { gave_up = WAIT_cache_q; return false; }
      if (elect_one()) {
        const CaSeg &s = segs[seg % CA_RING];
        mbar_expect_tx(q_full + qb, (uint32_t)(a.tile_rows * a.group * 128 * KP));
        for (int kp = 0; kp < KP; ++kp) tma_load_5d(q_s + qb * Sh::Q_BYTES + kp * Sh::Q_PANEL, &map_q, q_full + qb, 0, kp, 0, s.kvh, s.row0, pol);
      }
      __syncwarp();
      return true;
    };
    fetch(0);
    int seg = 0;
    for (int n; !gave_up && (n = segment(seg, WAIT_cache_q)) > 0; ++seg) {
      const int qb = seg & 1;
      bool ahead = false;
      if (!mbar_wait_warp(q_full + qb, (uint32_t)(seg >> 1) & 1u, abort_flag)) { gave_up = WAIT_cache_q; break; }
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        if (!__all_sync(0xffffffffu, mbar_wait(s_empty + sb, sph, abort_flag) && mbar_wait(k_full + st, ph, abort_flag))) { gave_up = WAIT_cache_k; break; }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(tmem_base + (uint32_t)(sb * CF_N), kd + (uint64_t)((st * Sh::STAGE + kp * Sh::PANEL + k * 32) >> 4),
                       qd + (uint64_t)((qb * Sh::Q_BYTES + kp * Sh::Q_PANEL + k * 32) >> 4), idesc, (kp > 0 || k > 0) ? 1u : 0u);
          mma_commit(k_empty + st);
          mma_commit(s_full + sb);
          if (i == n - 1) mma_commit(q_empty + qb);
        }
        __syncwarp();
        if (++st == STAGES) { st = 0; ph ^= 1u; }
        if (++sb == CF_S) { sb = 0; sph ^= 1u; }
        // the next segment's, as soon as it is known and there is room; the producer has left it by the time this one's last keys have come
        if (!ahead) {
          const int nx = seg + 1;
          const bool now = i == n - 1 || (mbar_test(seg_full + nx % CA_RING, (uint32_t)(nx / CA_RING) & 1u) && mbar_test(q_empty + (nx & 1), (uint32_t)(nx >> 1 & 1) ^ 1u));
          if (__all_sync(0xffffffffu, now)) {
            ahead = true;
            if (!fetch(nx)) break;
          }
        }
      }
    }
    for (int i = 0; i < 2 && !gave_up; ++i, ++seg)          // the last releases of the queries
      if (!mbar_wait_warp(q_empty + (seg & 1), (uint32_t)(seg >> 1 & 1) ^ 1u, abort_flag)) gave_up = WAIT_cache_last;
  } else if (warp == 2) {
    // ------------------------------------------------------------------ O^T += V^T P^T
    constexpr uint32_t idesc = (1u << 4) | CaType<T>::IDESC | (1u << 15) | ((uint32_t)(CF_N >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t vd = smem_desc_mn(smem_u32(v_s), Sh::PANEL), pd = smem_desc(smem_u32(p_s));
    int st = 0, g = 0;
    uint32_t ph = 0;
    for (int seg = 0, n; (n = segment(seg, WAIT_cache_o)) > 0; ++seg) {
      const int ob = seg & 1;
      if (seg > 1 && !mbar_wait_warp(o_free + ob, (uint32_t)((seg >> 1) - 1) & 1u, abort_flag)) { gave_up = WAIT_cache_o; break; }
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        const int pb = g & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(v_full + st, ph, abort_flag) && mbar_wait(p_full + pb, (uint32_t)(g >> 1) & 1u, abort_flag))) { gave_up = WAIT_cache_p_v; break; }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int mt = 0; mt < Sh::MT; ++mt)
#pragma unroll
            for (int k = 0; k < BLK / 16; ++k)                              // 16 keys: two groups of eight rows of V, 32 bytes of a row of P
              mma_bf16(o_base + (uint32_t)(ob * Sh::O_COLS + mt * CF_N), vd + (uint64_t)((st * Sh::STAGE + mt * 2 * Sh::PANEL + k * 2048) >> 4),
                       pd + (uint64_t)((pb * Sh::P_BYTES + (k >> 2) * Sh::P_PANEL + (k & 3) * 32) >> 4), idesc, (i > 0 || k > 0) ? 1u : 0u);
          mma_commit(v_empty + st);
          mma_commit(o_done + pb);
        }
        __syncwarp();
        if (++st == STAGES) { st = 0; ph ^= 1u; }
      }
      if (gave_up) break;
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ softmax: a key of the unit per thread; epilogue: a channel per thread
    const int q = warp & 3, t = q * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(q * 32) << 16;
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity, uint64_t *bar2 = nullptr, uint32_t parity2 = 0) {      // one lane polls for the warp, where it has to wait at all
      if (__all_sync(0xffffffffu, ok && mbar_test(bar, parity) && (!bar2 || mbar_test(bar2, parity2)))) return;
      int v = 1;
      if (lane == 0 && (!ok || !mbar_wait(bar, parity, abort_flag) || (bar2 && !mbar_wait(bar2, parity2, abort_flag)))) v = 0;
      if (!__shfl_sync(0xffffffffu, v, 0) && ok) {
        ok = false;
        if (lane == 0) wait_expired(status, WAIT_cache_softmax, abort_flag, -1);
      }
    };
    const float scale = a.scale_log2;
    const bool tree = !PAGES && a.tree, has_key = t < BLK;
    const uint32_t p_row = (uint32_t)((t >> 6) * Sh::P_PANEL + (t & 7) * 2), p_chunk = (uint32_t)(t & 63) >> 3;      // where the key stands in a row of P
    int g = 0, sb = 0;
    uint32_t sph = 0;
    for (int seg = 0;; ++seg) {
      const int n = segment(seg, WAIT_cache_softmax), ob = seg & 1;
      const CaSeg &s = segs[seg % CA_RING];
      const int n_e = n > 0 ? s.rows * a.group : 0;
      // the entries' rows, and what they see: keys below vis (counted from the segment's first), in a tree their own ones as the mask has them
      if (n > 0 && t < NE) {
        const int r = s.row0 + min(t, n_e - 1) / a.group;
        int vis = 0x7fffffff, nodes = 128;                  // (own keys end with the nodes anyway, shared ones do not)
        if (!PAGES && t < n_e && (s.phase || plan.partial)) {
          int tail0 = s.tail0, q0 = s.q0;
          if (!s.phase) {
            const CaSeq sq(a, ca_seq_of(a, r));
            tail0 = sq.len - sq.n;
            q0 = sq.q0;
            nodes = min(sq.n, 128);
          }
          vis = tail0 + (tree ? 0 : r - q0 + 1) - (s.key0 + s.b0 * BLK);
        }
        e_vis[ob][t] = vis;
        e_row[ob][t] = r;
        e_nodes[ob][t] = nodes;
      }
      if (cf_any(n <= 0)) break;                            // (whatever a wait of one warp came to, they all go on or all leave: barriers follow)
      int least = e_vis[ob][0];                             // what every entry sees
#pragma unroll
      for (int e = 1; e < NE; ++e) least = min(least, e_vis[ob][e]);
      float m_ref[NE], l[NE], l_true[NE];
#pragma unroll
      for (int e = 0; e < NE; ++e) { m_ref[e] = -INFINITY; l[e] = l_true[e] = 0.f; }
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        const int pb = g & 1;
        // S of the unit, and room for its P: O of the unit before last (its barrier's phases are all waited for, one behind the other)
        wait(s_full + sb, sph, g > 1 ? o_done + pb : nullptr, (uint32_t)((g >> 1) - 1) & 1u);
        tc_fence_after();
        uint32_t sr[NE];
        cf_ld(tmem_base + lane_addr + (uint32_t)(sb * CF_N), sr);
        const uint4 um = masks[g % CA_RING];
        const bool all = least - i * BLK >= BLK && (um.x & um.y & (BLK == 128 ? um.z & um.w : 0xffffffffu)) == 0xffffffffu;
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_empty + sb);
        if (++sb == CF_S) { sb = 0; sph ^= 1u; }
        float x[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) x[e] = __uint_as_float(sr[e]);
        bool there = has_key;
        if (!all) {
          const uint32_t mw = q == 0 ? um.x : q == 1 ? um.y : q == 2 ? um.z : um.w;
          there = has_key && (mw >> lane & 1u);
          uint32_t sees = 0;
          if (!tree) {
#pragma unroll
            for (int e = 0; e < NE; ++e) sees |= (uint32_t)(t + i * BLK < e_vis[ob][e]) << e;
          } else {
#pragma unroll 1
            for (int e = 0; e < n_e; ++e) {
              const int node = t + i * BLK - e_vis[ob][e];                  // of the key
              if (node < 0 || (node < e_nodes[ob][e] && a.tree[(long long)e_row[ob][e] * 4 + (node >> 5)] >> (node & 31) & 1u)) sees |= 1u << e;
            }
          }
#pragma unroll
          for (int e = 0; e < NE; ++e) x[e] = there && (sees >> e & 1u) ? x[e] : -INFINITY;
        }
        bool grow = false;
#pragma unroll
        for (int e = 0; e < NE; ++e) grow = grow || (e < n_e && x[e] * scale > m_ref[e] + CaType<T>::RESCALE);
        if (cf_any(grow && has_key)) {
          // ---- the maxima of the unit, and new references where they have grown
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const float v = order_value(__reduce_max_sync(0xffffffffu, order_key(has_key ? x[e] : -INFINITY)));
            if (lane == 0) red[q][e] = v;
          }
          cf_sync();
          float corr[NE];
#pragma unroll
          for (int e = 0; e < NE; ++e) {                                    // (entries past n_e have scores of nothing in particular, and nobody reads what comes of them)
            const float bm = fmaxf(fmaxf(red[0][e], red[1][e]), fmaxf(red[2][e], red[3][e])) * scale;
            const bool more = bm > m_ref[e] + CaType<T>::RESCALE;
            corr[e] = more ? ex2(m_ref[e] - bm) : 1.f;
            l[e] *= corr[e]; l_true[e] *= corr[e];
            m_ref[e] = more ? bm : m_ref[e];
          }
          if (i > 0) {                                                      // behind the O of every earlier unit
            wait(o_done + ((g - 1) & 1), (uint32_t)((g - 1) >> 1) & 1u);
            tc_fence_after();
#pragma unroll
            for (int mt = 0; mt < Sh::MT; ++mt) {
              uint32_t o[NE];
              const uint32_t at = o_base + lane_addr + (uint32_t)(ob * Sh::O_COLS + mt * CF_N);
              cf_ld(at, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < NE; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * corr[e]);
              cf_st(at, o);
            }
            tmem_st_wait();
          }
        }
        if (has_key) {
          uint8_t *p = p_s + pb * Sh::P_BYTES + p_row;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
              const float w_true = ex2(fmaf(x[e], scale, (m_ref[e] == -INFINITY ? 0.f : -m_ref[e]) + CaType<T>::SHIFT));
              const T w = from_f<T>(w_true);
              *reinterpret_cast<T *>(p + e * 128 + ((p_chunk ^ (e & 7)) << 4)) = w;
              l[e] += to_f(w);
              l_true[e] += w_true;
            }
          if (!all && !there) {
            // values that are nobody's may be anything, and 0 times that not 0
            mbar_wait(v_full + g % STAGES, (uint32_t)(g / STAGES) & 1u, abort_flag);
            uint8_t *v = v_s + (g % STAGES) * Sh::STAGE + t * 128;
#pragma unroll
            for (int kp = 0; kp < KP; ++kp)
#pragma unroll
              for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4 *>(v + kp * Sh::PANEL + c * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + pb);
      }
      // ---- epilogue.  The sums of weights, across the lanes by halves: lane e (32 / NE) ends up with those of entry e
      {
        float v[NE], u[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) { v[e] = l[e]; u[e] = l_true[e]; }
        int width = NE;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          if (width > 1) {
            width /= 2;
            const bool up = (lane & o) != 0;
#pragma unroll
            for (int j = 0; j < NE / 2; ++j)
              if (j < width) {
                v[j] = (up ? v[j + width] : v[j]) + __shfl_xor_sync(0xffffffffu, up ? v[j] : v[j + width], o);
                u[j] = (up ? u[j + width] : u[j]) + __shfl_xor_sync(0xffffffffu, up ? u[j] : u[j + width], o);
              }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
            u[0] += __shfl_xor_sync(0xffffffffu, u[0], o);
          }
        }
        if (lane % (32 / NE) == 0) sums[q][lane / (32 / NE)] = make_float2(v[0], u[0]);
      }
#pragma unroll
      for (int e = 0; e < NE; ++e) if (t == e) refs[e] = m_ref[e];
      cf_sync();
      // a thread per entry: what the segment leaves of it, and where its O goes
      const bool final = s.b0 == 0 && !s.follow && (PAGES || !plan.shared);
      if (t < n_e && t < NE) {
        const float2 s0 = sums[0][t], s1 = sums[1][t], s2 = sums[2][t], s3 = sums[3][t];
        const float sl = (s0.x + s1.x) + (s2.x + s3.x), st = (s0.y + s1.y) + (s2.y + s3.y), m = refs[t] == -INFINITY ? refs[t] : refs[t] - CaType<T>::SHIFT;
        const int r = e_row[ob][t], h = s.kvh * a.group + t % a.group;
        const bool starts = s.b0 == 0, row_on = !PAGES || s.seq >= 0;
        const long long rh = (long long)r * a.heads + h, at = starts ? (PAGES ? rh : (long long)s.phase * a.rows * a.heads + rh) : (long long)(a.cont_base + cta) * 128 + t;
        if (starts) {
          a.part_ml[at] = make_float4(m, sl, st, pack_follow(t, final || !row_on ? CA_DONE : s.follow, a.cont_base + cta + 1));
          if (final && row_on && a.lse) a.lse[rh] = sl > 0.f ? (m + log2f(st)) * 0.6931471805599453f : -INFINITY;
        } else a.cont_ml[at] = make_float4(m, sl, st, 0.f);
        e_to[t] = final ? (row_on ? (void *)((T *)a.out + r * a.out_ld + (long long)h * HD) : nullptr) : (void *)((starts ? a.part_o : a.cont_o) + at * HD);
        e_inv[t] = sl > 0.f ? 1.f / sl : 0.f;
      }
      wait(o_done + ((g - 1) & 1), (uint32_t)((g - 1) >> 1) & 1u);
      tc_fence_after();
      uint32_t o[Sh::MT][NE];
#pragma unroll
      for (int mt = 0; mt < Sh::MT; ++mt) cf_ld(o_base + lane_addr + (uint32_t)(ob * Sh::O_COLS + mt * CF_N), o[mt]);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free + ob);
      cf_sync();
      if (t < HD && ok) {
#pragma unroll
        for (int e = 0; e < NE; ++e)
          if (e < n_e) {
            void *to = e_to[e];
#pragma unroll
            for (int mt = 0; mt < Sh::MT; ++mt) {
              if (!final) ((float *)to)[mt * 128 + t] = __uint_as_float(o[mt][e]);
              else if (to) ((T *)to)[mt * 128 + t] = from_f<T>(__uint_as_float(o[mt][e]) * e_inv[e]);
            }
          }
      }
    }
    // the last O but one: nobody has waited for its arrival
    if (g > 1) wait(o_done + (g & 1), (uint32_t)((g - 2) >> 1) & 1u);
  }
  if (gave_up && lane == 0) wait_expired(status, gave_up, abort_flag, -1);
  drain_if_aborted(abort_flag);
  if (a.early) pdl_wait();                   // the end of this launch is the end of both
  pdl_trigger();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
  }
}
