// Attention over a paged cache that a program holds itself, on the tcgen05 tensor cores: a ragged batch whose sequences may begin with the
// same pages (dream_cache_attn), and rows that read listed pages (dream_cache_attn_pages).
//
// Where a tile has more than four query entries; for fewer see cache_few.cuh, and for how the work is dealt out cache_work.cuh.
//
// A segment.  S = Q K^T (128 x 128 keys, 64 at head_dim 256; fp32 in TMEM, three or four buffers), softmax by sixteen warps: a group of 16 rows has two, one for each half of the unit's
// keys, and the four lanes of a quad share a row (and the one eight further on).  One pass with a running reference m that follows the
// row's maximum only when that has outgrown it (the accumulator is then rescaled, seldom; whether it has is one barrier with a vote between the two warps), P = 2^(s - m)
// rounded to the cache's type into the columns the scores came from, O += P V with P as the TMEM operand.  l sums the rounded P, so that the weights add up to 1 whatever their rounding, which
// then moves the result by at most half a step of sum w |v - out| (against 64 bits 1.7e-3 to 2.2e-3 of the norm in bf16, most behind long contexts, and 2.9e-4 in fp16; with weights of 32 bits 1.6e-3 and 2.1e-4,
// for twice the product with V); the log-sum-exp has a sum of its own, of P as it was.  K and V come by TMA in two rings that
// run on from segment to segment, so that the next one's keys are under way while one ends.  The producer of K alone says what the segments are, ahead of
// everybody else, and leaves them in a ring in shared memory.
// Bound by the length of that chain per unit (S read, maxima, vote, exponentials, P written), 2200 cycles at 64 columns and 1500 or more at 256, where the products are 512 and 1024: seven prompts of 500 tokens
// behind 4096, 16 heads over 8 of 256, 157 us, the tensor pipe busy 46 % of it.  One CTA to an SM: with units of 64 keys, eight softmax warps and two CTAs a prompt of
// 4096 at 128 columns took 208 us in place of 153, 1500 rows behind 4096 at 256 196 in place of 174.
// Warps: 0 K and segments, 1 Q, S and TMEM, 2 O, 3 V, 4..19 softmax and epilogue.
#pragma once
#include "attn_tc.cuh"
#include "cache_work.cuh"

#define CA_SOFTMAX 16                    // softmax warps
#define CA_THREADS (128 + 32 * CA_SOFTMAX)

template <int HD> struct CaShape {
  static constexpr int BLK = HD == 256 ? 64 : 128;                     // keys of a unit
  static constexpr int KP = HD / 64;                                   // 64-column panels of a row
  static constexpr int STAGES = HD == 64 ? 5 : 2;                      // units of K (and of V) in shared memory
  static constexpr int S_BUFS = HD == 64 ? 3 : HD == 128 ? 3 : 4;      // what the 512 TMEM columns hold beside O
  static constexpr int TMEM_COLS = 512;
  static constexpr int Q_BYTES = 128 * HD * 2, Q_PANEL = 128 * 128;
  static constexpr int STAGE = BLK * HD * 2, PANEL = BLK * 128;
  static constexpr size_t SMEM = 1024 + Q_BYTES + 2 * STAGES * STAGE + 2048;
};

// D += A B with A in TMEM (lane = row, a column holds two neighbouring elements of K).
__device__ __forceinline__ void mma_tmem_a(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accum) : "memory");
}
// 16 lanes x 32 columns, as tmem_ld16x64 has them.
__device__ __forceinline__ void tmem_ld16x32(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
}
// 16 lanes x 16 columns: lane 4 i + j of the warp puts r[2 c] into column 4 c + j of TMEM lane i, r[2 c + 1] into that of lane i + 8.
__device__ __forceinline__ void tmem_st16x16(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_st16x32f(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// Two at a time (an instruction for both).
__device__ __forceinline__ float2 ca_add(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(r)) : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
  return r;
}
__device__ __forceinline__ float2 ca_fma(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long &>(r)) : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)), "l"(reinterpret_cast<unsigned long long &>(c)));
  return r;
}

// Eight floats to a 32-byte boundary: even columns in x, odd ones in y.  (Four lanes store a whole line: in pieces of eight bytes a tile's partial result took 4000 cycles.)
__device__ __forceinline__ void st_global8(float *p, const uint32_t (&x)[4], const uint32_t (&y)[4]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(x[0]), "r"(y[0]), "r"(x[1]), "r"(y[1]), "r"(x[2]), "r"(y[2]), "r"(x[3]), "r"(y[3]) : "memory");
}
// The barrier of a pair of softmax warps, with and without a vote.
__device__ __forceinline__ bool ca_any(int pair, bool mine) {
  uint32_t r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %2, 0;\n barrier.cta.red.or.pred q, %1, 64, p;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(r) : "r"(1 + pair), "r"((uint32_t)mine) : "memory");
  return r != 0;
}
__device__ __forceinline__ void ca_sync(int pair) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(1 + pair) : "memory"); }

template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(CA_THREADS, 1)
k_cache_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
             const __grid_constant__ CUtensorMap map_q_small, const __grid_constant__ CacheAttnArgs a) {
  using Sh = CaShape<HD>;
  constexpr int STAGES = Sh::STAGES, KP = Sh::KP, SB = Sh::S_BUFS, BLK = Sh::BLK;
  extern __shared__ uint8_t ca_smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)ca_smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *q_s = smem, *k_s = q_s + Sh::Q_BYTES, *v_s = k_s + STAGES * Sh::STAGE;
  uint64_t *bars = (uint64_t *)(v_s + STAGES * Sh::STAGE);
  uint64_t *k_full = bars, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES;
  uint64_t *s_full = v_empty + STAGES, *p_full = s_full + SB, *o_done = p_full + SB, *q_full = o_done + SB, *o_free = q_full + 1, *seg_full = o_free + 1;
  uint4 *masks = (uint4 *)(((uintptr_t)(seg_full + CA_RING) + 15) & ~(uintptr_t)15);                         // [CA_RING] which keys of a unit there are
  CaSeg *segs = (CaSeg *)(masks + CA_RING);                                // [CA_RING]
  uint32_t *tmem_base_p = (uint32_t *)(segs + CA_RING);
  volatile int *abort_flag = (volatile int *)(tmem_base_p + 1);
  __shared__ CaPlanShared plan;
  __shared__ int sh_status[2];
  __shared__ float pair_max[CA_SOFTMAX / 2][2][16];                        // what the halves of a pair tell each other: maxima of their rows ...
  __shared__ float2 pair_sum[CA_SOFTMAX / 2][2][16];                       // ... and sums of weights

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, cta = blockIdx.x;
  if (a.early) {                             // no sequence has more entries than the other kernel's tiles: there is nothing to set up, and what follows need not wait for it
    bool some = false;
    for (int i = threadIdx.x; i < a.c.n_seqs; i += CA_THREADS) some = some || CaSeq(a, i).taken(a);
    if (!__syncthreads_or(some)) {
      pdl_trigger();
      pdl_wait();
      return;
    }
  }
  unsigned long long *tr = trace_open();
  if (warp == 0) {
    if (lane < STAGES) { mbar_init(k_full + lane, 1); mbar_init(k_empty + lane, 1); mbar_init(v_full + lane, 1); mbar_init(v_empty + lane, 1); }
    else if (lane >= 8 && lane < 8 + SB) { mbar_init(s_full + lane - 8, 1); mbar_init(p_full + lane - 8, CA_SOFTMAX); mbar_init(o_done + lane - 8, 1); }
    else if (lane >= 16) mbar_init(seg_full + lane - 16, 1);
    if (lane == 12) { mbar_init(q_full, 1); mbar_init(o_free, CA_SOFTMAX); *abort_flag = 0; }
    else if (lane == 13) { plan.partial = plan.longest = 0; sh_status[0] = sh_status[1] = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q_small) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_p)), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  static_assert(CA_RING == 16, "a lane inits each of the segments' barriers");
  static_assert(CA_RING > STAGES + SB + 1, "what the producer leaves is read until a unit's P is done");
  static_assert(sizeof(uint64_t) * (4 * STAGES + 3 * SB + 2 + CA_RING) + 16 + sizeof(uint4) * CA_RING + sizeof(CaSeg) * CA_RING + 8 <= 2048, "room for the barriers and rings");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (!a.early) pdl_wait();
  if (a.let) pdl_trigger();
  trace_stamp(tr, TR_k_cache_attn);
  int *status = a.status ? a.status : sh_status;

  CaWalk<BLK, 1, PAGES> w;
  w.plan(a, plan, status);
  const uint32_t tmem_base = *tmem_base_p;
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
    // ------------------------------------------------------------------ queries, and S = Q K^T: both operands K-major, N = BLK
    constexpr uint32_t idesc = (1u << 4) | CaType<T>::IDESC | ((uint32_t)(BLK >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t qd = smem_desc(smem_u32(q_s)), kd = smem_desc(smem_u32(k_s));
    const uint32_t s_addr = tmem_base + HD;
    const uint64_t pol = policy_evict_normal();
    int ks = 0, g = 0, sb = 0;
    uint32_t kph = 0, sph = 1;                              // sph: parity of the buffer's last O (1: none yet)
    for (int seg = 0, n; (n = segment(seg, WAIT_cache_q)) > 0; ++seg) {
      if (elect_one()) {
        const CaSeg &s = segs[seg % CA_RING];
        const bool small = s.rows <= a.q_small;
        mbar_expect_tx(q_full, (uint32_t)((small ? a.q_small : a.tile_rows) * a.group * 128 * KP));
        for (int kp = 0; kp < KP; ++kp) tma_load_5d(q_s + kp * Sh::Q_PANEL, small ? &map_q_small : &map_q, q_full, 0, kp, 0, s.kvh, s.row0, pol);
      }
      __syncwarp();
      if (!mbar_wait_warp(q_full, (uint32_t)seg & 1u, abort_flag)) { gave_up = WAIT_cache_q; break; }
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        if (!__all_sync(0xffffffffu, mbar_wait(o_done + sb, sph, abort_flag) && mbar_wait(k_full + ks, kph, abort_flag))) { gave_up = WAIT_cache_k; break; }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16(s_addr + (uint32_t)(sb * BLK), qd + (uint64_t)((kp * Sh::Q_PANEL + k * 32) >> 4),
                       kd + (uint64_t)((ks * Sh::STAGE + kp * Sh::PANEL + k * 32) >> 4), idesc, (kp > 0 || k > 0) ? 1u : 0u);
          mma_commit(k_empty + ks);
          mma_commit(s_full + sb);
        }
        __syncwarp();
        if (++ks == STAGES) { ks = 0; kph ^= 1u; }
        if (++sb == SB) { sb = 0; sph ^= 1u; }
      }
      if (gave_up) break;
      // the next queries take these ones' place when S of the last unit is done
      if (!mbar_wait_warp(s_full + (g - 1) % SB, (uint32_t)((g - 1) / SB) & 1u, abort_flag)) { gave_up = WAIT_cache_k; break; }
    }
    // the last O of each buffer: the softmax waits for that of a segment's last unit, and for the others' arrivals nobody does
#pragma unroll 1
    for (int i = 0; i < SB && !gave_up; ++i) {
      if (!mbar_wait_warp(o_done + sb, sph, abort_flag)) gave_up = WAIT_cache_last;
      if (++sb == SB) { sb = 0; sph ^= 1u; }
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------ O += P V: P in TMEM, V MN-major, N = head_dim
    constexpr uint32_t idesc = (1u << 4) | CaType<T>::IDESC | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t vd = smem_desc_mn(smem_u32(v_s), Sh::PANEL);
    const uint32_t p_addr = tmem_base + HD;
    int vs = 0, g = 0, sb = 0;
    uint32_t vph = 0, pph = 0;
    for (int seg = 0, n; (n = segment(seg, WAIT_cache_o)) > 0; ++seg) {
      if (seg > 0 && !mbar_wait_warp(o_free, (uint32_t)(seg - 1) & 1u, abort_flag)) { gave_up = WAIT_cache_o; break; }
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        if (!__all_sync(0xffffffffu, mbar_wait(v_full + vs, vph, abort_flag) && mbar_wait(p_full + sb, pph, abort_flag))) { gave_up = WAIT_cache_p_v; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t bd = vd + (uint64_t)((vs * Sh::STAGE) >> 4);
#pragma unroll
          for (int k = 0; k < BLK / 16; ++k)                             // 16 keys: eight columns of P, two groups of eight rows of V
            mma_tmem_a(tmem_base, p_addr + (uint32_t)(sb * BLK + k * 8), bd + (uint64_t)(k * 128), idesc, (i > 0 || k > 0) ? 1u : 0u);
          mma_commit(v_empty + vs);
          mma_commit(o_done + sb);
        }
        __syncwarp();
        if (++vs == STAGES) { vs = 0; vph ^= 1u; }
        if (++sb == SB) { sb = 0; pph ^= 1u; }
      }
      if (gave_up) break;
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------ softmax and epilogue: 16 rows of the tile have a warp for the first half of a unit's keys
    // and one for the second; a lane has a quarter of the half's keys for two rows
    constexpr int NC = BLK / 64;                            // runs of 32 keys in a half
    const int ws = warp - 4, half = ws >> 3, pair = ws & 7, base = (warp & 3) * 32 + (ws & 4 ? 16 : 0), quad = lane >> 2, ql = lane & 3;
    const uint32_t lane_addr = tmem_base + ((uint32_t)base << 16);
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) {                       // one lane polls for the warp, where it has to wait at all (64 readers of 32768 keys, 64 wide: 92 -> 87 us)
      if (__all_sync(0xffffffffu, ok && mbar_test(bar, parity))) return;
      int v = 1;
      if (lane == 0 && (!ok || !mbar_wait(bar, parity, abort_flag))) v = 0;
      if (!__shfl_sync(0xffffffffu, v, 0) && ok) {
        ok = false;
        if (lane == 0) wait_expired(status, WAIT_cache_softmax, abort_flag, -1);
      }
    };
    const float scale = a.scale_log2;
    const bool tree = !PAGES && a.tree;
    int g = 0, sb = 0;
    uint32_t sph = 0;
    for (int seg = 0;; ++seg) {
      const int n = segment(seg, WAIT_cache_softmax);
      if (ca_any(pair, n <= 0)) break;                      // (whatever a wait of one of the two came to, both go on or both leave: barriers follow)
      const CaSeg &s = segs[seg % CA_RING];                 // read where it is needed: registers are short
      const int n_entries = s.rows * a.group;
      const bool active = base < n_entries, mine[2] = {base + quad < n_entries, base + quad + 8 < n_entries};
      // a row sees the keys below vis (counted from this half of the segment's first unit), and in a tree its own ones as the mask has them
      int vis[2] = {0x7fffffff, 0x7fffffff};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (!PAGES && mine[k] && (s.phase || plan.partial)) {
          const int r = s.row0 + (base + quad + 8 * k) / a.group;
          int tail0 = s.tail0, q0 = s.q0;
          if (!s.phase) {                                                   // the sequence that has the row
            const CaSeq q(a, ca_seq_of(a, r));
            tail0 = q.len - q.n;
            q0 = q.q0;
          }
          vis[k] = tail0 + (tree ? 0 : r - q0 + 1) - (s.key0 + s.b0 * BLK) - half * (BLK / 2);
        }
      }
      float m_ref[2] = {-INFINITY, -INFINITY};
      float2 l2[2], t2[2];                                                  // this lane's share of the sums, rounded and as they were
      l2[0] = l2[1] = t2[0] = t2[1] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        wait(s_full + sb, sph);
        const uint4 um4 = masks[g % CA_RING];
        if ((um4.x & um4.y & (BLK > 64 ? um4.z & um4.w : 0xffffffffu)) != 0xffffffffu) {
          // values that are nobody's may be anything, and 0 times that not 0: all the warps' lanes, some to a key.  With fewer stages than buffers of S a unit's scores may be here before
          // the values of the unit STAGES back, and then the parity of their barrier is that of the unit before that one; behind its O it says what it is asked
          constexpr int LANES = 32 * CA_SOFTMAX / BLK;
          const int key = (ws * 32 + lane) / LANES, word = key >> 5;
          if (!((word == 0 ? um4.x : word == 1 ? um4.y : word == 2 ? um4.z : um4.w) >> (key & 31) & 1u) &&
              (STAGES >= SB || g < STAGES || mbar_wait(o_done + (g - STAGES) % SB, (uint32_t)((g - STAGES) / SB) & 1u, abort_flag)) &&
              mbar_wait(v_full + g % STAGES, (uint32_t)(g / STAGES) & 1u, abort_flag)) {
            uint8_t *v = v_s + (g % STAGES) * Sh::STAGE + key * 128;
#pragma unroll 1
            for (int j = lane % LANES; j < KP * 8; j += LANES) *reinterpret_cast<uint4 *>(v + (j >> 3) * Sh::PANEL + (j & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();
        }
        if (active) {
          tc_fence_after();
          const uint32_t s_col = lane_addr + (uint32_t)(HD + sb * BLK);
          uint32_t sr[NC][16];                                              // sr[x][4 c + 2 k + j]: row k, key 32 x + 8 c + 2 ql + j of the half
#pragma unroll
          for (int x = 0; x < NC; ++x) tmem_ld16x32(s_col + (uint32_t)(half * (BLK / 2) + x * 32), sr[x]);
          uint32_t um[NC];
          um[0] = NC == 2 ? (half ? um4.z : um4.x) : (half ? um4.y : um4.x);
          if (NC == 2) um[NC - 1] = half ? um4.w : um4.y;
          const int left0 = vis[0] - i * BLK, left1 = vis[1] - i * BLK;
          const bool all = (um[0] & um[NC - 1]) == 0xffffffffu && left0 >= BLK / 2 && left1 >= BLK / 2;
          tmem_ld_wait();
          if (!__all_sync(0xffffffffu, all)) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int x = 0; x < NC; ++x) {
                const int left = (k ? left1 : left0) - 32 * x;
                uint32_t m = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                if (tree && left < 32 && mine[k]) {
                  const uint32_t *t = a.tree + (long long)(s.row0 + (base + quad + 8 * k) / a.group) * 4;
                  const int sh = -left, word = sh >> 5;                     // node of the first key; in front of the nodes: the bits come later
                  const uint32_t w0 = word >= 0 && word < 4 ? t[word] : 0u, w1 = word >= -1 && word < 3 ? t[word + 1] : 0u;
                  m |= __funnelshift_r(w0, w1, sh & 31);
                  if (!s.phase) {                                           // (shared pages do not end where the row's sequence does: no bits past its nodes)
                    const int past = left + CaSeq(a, ca_seq_of(a, s.row0 + (base + quad + 8 * k) / a.group)).n;
                    m &= past >= 32 ? 0xffffffffu : past > 0 ? (1u << past) - 1u : 0u;
                  }
                }
                m = (m & um[x]) >> (2 * ql);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  sr[x][4 * c + 2 * k] = m >> (8 * c) & 1u ? sr[x][4 * c + 2 * k] : 0xff800000u;
                  sr[x][4 * c + 2 * k + 1] = m >> (8 * c) & 2u ? sr[x][4 * c + 2 * k + 1] : 0xff800000u;
                }
              }
          }
          float bm[2];
          bool grow = false;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float x = -INFINITY;
#pragma unroll
            for (int y = 0; y < NC; ++y)
#pragma unroll
              for (int c = 0; c < 4; ++c) x = fmaxf(x, fmaxf(__uint_as_float(sr[y][4 * c + 2 * k]), __uint_as_float(sr[y][4 * c + 2 * k + 1])));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            bm[k] = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2)) * scale;
            grow = grow || (mine[k] && bm[k] > m_ref[k] + CaType<T>::RESCALE);
          }
          // (and behind the vote both halves have their scores: P may take the columns of the first half's)
          if (ca_any(pair, grow)) {
            // the two halves' maxima; the accumulator takes the new reference, behind the O of every earlier unit, each half one half of its columns
            if (ql == 0) { pair_max[pair][half][quad] = bm[0]; pair_max[pair][half][quad + 8] = bm[1]; }
            ca_sync(pair);
            float corr[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float x = fmaxf(bm[k], pair_max[pair][half ^ 1][quad + 8 * k]);
              const bool more = mine[k] && x > m_ref[k] + CaType<T>::RESCALE;
              corr[k] = more ? ex2(m_ref[k] - x) : 1.f;
              l2[k].x *= corr[k]; l2[k].y *= corr[k]; t2[k].x *= corr[k]; t2[k].y *= corr[k];
              m_ref[k] = more ? x : m_ref[k];
            }
            if (i > 0) {
              wait(o_done + (g - 1) % SB, (uint32_t)((g - 1) / SB) & 1u);
              tc_fence_after();
#pragma unroll 1
              for (int c0 = half * (HD / 2); c0 < (half + 1) * (HD / 2); c0 += 32) {
                uint32_t o[16];
                tmem_ld16x32(lane_addr + (uint32_t)c0, o);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * (c & 2 ? corr[1] : corr[0]));
                tmem_st16x32f(lane_addr + (uint32_t)c0, o);
              }
            }
          }
#pragma unroll
          for (int x = 0; x < NC; ++x) {
            uint32_t p[8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float nbase = (m_ref[k] == -INFINITY ? 0.f : -m_ref[k]) + CaType<T>::SHIFT;
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const float2 d = ca_fma(make_float2(__uint_as_float(sr[x][4 * c + 2 * k]), __uint_as_float(sr[x][4 * c + 2 * k + 1])), make_float2(scale, scale), make_float2(nbase, nbase));
                const float2 w = make_float2(ex2(d.x), ex2(d.y));
                p[2 * c + k] = pack2(w.x, w.y, T());
                l2[k] = ca_add(l2[k], unpack2(p[2 * c + k], T()));
                t2[k] = ca_add(t2[k], w);
              }
            }
            tmem_st16x16(s_col + (uint32_t)(half * (BLK / 4) + x * 16), p);
          }
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + sb);
        if (++sb == SB) { sb = 0; sph ^= 1u; }
      }
      // ---- epilogue, each half one half of the columns
      float l[2], l_true[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        l[k] = l2[k].x + l2[k].y;
        l_true[k] = t2[k].x + t2[k].y;
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
        l_true[k] += __shfl_xor_sync(0xffffffffu, l_true[k], 1);
        l_true[k] += __shfl_xor_sync(0xffffffffu, l_true[k], 2);
        if (ql == 0) pair_sum[pair][half][quad + 8 * k] = make_float2(l[k], l_true[k]);
      }
      ca_sync(pair);
      const bool starts = s.b0 == 0, final = starts && !s.follow && (PAGES || !plan.shared), row_on = !PAGES || s.seq >= 0;
      float inv[2];
      long long at[2];
      int r[2], h[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float2 x = pair_sum[pair][0][quad + 8 * k], y = pair_sum[pair][1][quad + 8 * k];       // in this order in both
        l[k] = x.x + y.x;
        l_true[k] = x.y + y.y;
        inv[k] = l[k] > 0.f ? 1.f / l[k] : 0.f;
        const int e = base + quad + 8 * k;
        r[k] = s.row0 + e / a.group;
        h[k] = s.kvh * a.group + e % a.group;
        const long long rh = (long long)r[k] * a.heads + h[k];
        at[k] = starts ? (PAGES ? rh : (long long)s.phase * a.rows * a.heads + rh) : (long long)(a.cont_base + cta) * 128 + e;
        if (mine[k] && ql == 0 && half == 0) {
          const float m = m_ref[k] == -INFINITY ? m_ref[k] : m_ref[k] - CaType<T>::SHIFT;
          if (starts) {
            a.part_ml[at[k]] = make_float4(m, l[k], l_true[k], pack_follow(e, final || !row_on ? CA_DONE : s.follow, a.cont_base + cta + 1));
            if (final && row_on && a.lse) a.lse[rh] = l[k] > 0.f ? (m + log2f(l_true[k])) * 0.6931471805599453f : -INFINITY;
          } else a.cont_ml[at[k]] = make_float4(m, l[k], l_true[k], 0.f);
        }
      }
      wait(o_done + (g - 1) % SB, (uint32_t)((g - 1) / SB) & 1u);
      if (active && ok) {
        tc_fence_after();
#pragma unroll 1
        for (int c0 = half * (HD / 2); c0 < (half + 1) * (HD / 2); c0 += 32) {
          uint32_t o[16];                                                   // o[4 c + 2 k + j]: row k, column c0 + 8 c + 2 ql + j
          tmem_ld16x32(lane_addr + (uint32_t)c0, o);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t z[4], y[4];                                            // turned within the quad, a lane has eight columns that stand side by side
            if (final) {
#pragma unroll
              for (int c = 0; c < 4; ++c) z[c] = pack2(__uint_as_float(o[4 * c + 2 * k]) * inv[k], __uint_as_float(o[4 * c + 2 * k + 1]) * inv[k], T());
              quad_transpose(z, lane);
              if (mine[k] && row_on) *reinterpret_cast<uint4 *>((T *)a.out + (long long)r[k] * a.out_ld + (long long)h[k] * HD + c0 + 8 * ql) = make_uint4(z[0], z[1], z[2], z[3]);
            } else {
#pragma unroll
              for (int c = 0; c < 4; ++c) { z[c] = o[4 * c + 2 * k]; y[c] = o[4 * c + 2 * k + 1]; }
              quad_transpose(z, lane);
              quad_transpose(y, lane);
              if (mine[k]) st_global8((starts ? a.part_o : a.cont_o) + at[k] * HD + c0 + 8 * ql, z, y);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free);
    }
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
