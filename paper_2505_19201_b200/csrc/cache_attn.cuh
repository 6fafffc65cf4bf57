// Attention over a paged cache that a program holds itself, on the tcgen05 tensor cores: a ragged batch whose sequences may begin with the
// same pages (dream_cache_attn), and rows that read listed pages (dream_cache_attn_pages).
//
// Work.  An item is up to 128 query entries (entry = (row, query head of one KV-head group)) against a run of keys of one KV head, cut into
// units of 64 keys.  Shared pages: the rows of all sequences stand together, in tiles of 128 entries, so that the prefix is read once for all of them (once per
// tile).  A sequence's own tokens: its rows, tile by tile.  Listed pages: one row.  The units of all items, one behind the other, are dealt out to
// the CTAs in equal contiguous ranges, by arithmetic on the lengths that each CTA does for itself (they are on the device), so long contexts
// with few rows fill the GPU and short ones do not leave a tail.  A range is a few segments, each in one item.  A segment leaves (m, l, O) of its keys; k_cache_merge adds up the
// segments of a row, always in the same order.  The segment that starts an item has its place by row and head, a CTA's continuation
// of an item the CTA's own.
//
// A segment.  S = Q K^T (128 x 64, fp32 in TMEM, two buffers), softmax by 128 threads, a row each: one pass with a running reference m that follows the
// row's maximum only when that has outgrown it (the accumulator is then rescaled, seldom), P = 2^(s - m) rounded to the cache's type into the columns
// its scores came from, O += P V with P as the TMEM operand.  l sums the rounded P, so that the weights add up to 1 whatever their rounding, which
// then moves the result by at most half a step of sum w |v - out|; the log-sum-exp has a sum of its own, of P as it was.  K and V come by TMA in two rings that
// run on from segment to segment, so that the next one's keys are under way while one ends; its queries are fetched before the accumulator is read out.
// Warps: 0 TMA, 1 matrix instructions and TMEM, 2..5 softmax and epilogue.
#pragma once
#include "attn_tc.cuh"
#include "cache_rows.cuh"

#define CA_THREADS 192
#define CA_BLK 64                        // keys of a unit
#define CA_MASKS 16                      // ring of the units' key masks: more than the K ring's stages and two

template <int HD> struct CaShape {
  static constexpr int KP = HD / 64;                                   // 64-column panels of a row
  static constexpr int STAGES = HD == 64 ? 5 : 2;                      // units of K (and of V) in shared memory
  static constexpr int TMEM_COLS = HD + 2 * CA_BLK <= 256 ? 256 : 512;
  static constexpr int CTAS_PER_SM = HD == 256 ? 1 : 2;                // one walks its keys while the other starts or ends a segment
  static constexpr int Q_BYTES = 128 * HD * 2, Q_PANEL = 128 * 128;
  static constexpr int STAGE = CA_BLK * HD * 2, PANEL = CA_BLK * 128;
  static constexpr size_t SMEM = 1024 + Q_BYTES + 2 * STAGES * STAGE + 512;
};

struct CacheAttnArgs {
  CacheView c;
  const void *q;
  long long q_ld, out_ld;
  void *out;
  float *lse;
  const int *q_start, *kv_len;             // dense: rows by sequence
  const uint32_t *tree;                    // dense: [rows][4], or null
  const int *row_seq, *row_pos, *ids;      // pages
  int budget, rows, heads, group, tile_rows;
  int shared_tokens;                       // dense: keys [0, shared_tokens) are everybody's
  float scale_log2;
  float *part_o;                           // [phase][row][head][HD]: what the segment that starts an item leaves ...
  float4 *part_ml;                         // [phase][row][head]: its (m, l, l before rounding, what follows: see pack_follow)
  float *cont_o;                           // [CTA][128][HD], [CTA][128]: the segments that continue one
  float4 *cont_ml;
  int n_ctas;
  int *status;
};

// What the merge has to know about the segments behind an item's first: how many, from which CTA on, and the row's entry in the tile.
#define CA_DONE 0x7ff                      // nothing is left to merge
__device__ __forceinline__ float pack_follow(int entry, int n, int cta) { return __int_as_float(entry | n << 7 | cta << 18); }

template <typename T> struct CaType;
// The rounded P keeps all its digits between the largest value of the type and its smallest normal one: fp16's range ends 2^-14 below 1, so its P are
// 2^10 times larger and the reference is followed sooner.
template <> struct CaType<bf16> { static constexpr float SHIFT = 0.f, RESCALE = 8.f; static constexpr uint32_t IDESC = (1u << 7) | (1u << 10); };
template <> struct CaType<f16> { static constexpr float SHIFT = 10.f, RESCALE = 4.f; static constexpr uint32_t IDESC = 0u; };
__device__ __forceinline__ uint32_t pack2(float x, float y, bf16) { __nv_bfloat162 h = __floats2bfloat162_rn(x, y); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ uint32_t pack2(float x, float y, f16) { __half2 h = __floats2half2_rn(x, y); return *reinterpret_cast<uint32_t *>(&h); }
__device__ __forceinline__ float2 unpack2(uint32_t w, bf16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, f16) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

// D += A B with A in TMEM (lane = row, a column holds two neighbouring elements of K).
__device__ __forceinline__ void mma_tmem_a(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accum) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31]) : "memory");
}

// A sequence as the call gives it, held within the buffers whatever its numbers say.
struct CaSeq {
  int q0, n, len;                          // first row, rows, tokens
  __device__ __forceinline__ CaSeq(const CacheAttnArgs &a, int s) {
    q0 = min(max(a.q_start[s], 0), a.rows);
    n = min(max(a.q_start[s + 1], q0), a.rows) - q0;
    len = min(max(a.kv_len[s], 0), a.c.pages_per_seq << a.c.page_shift);
  }
  __device__ __forceinline__ int tiles(const CacheAttnArgs &a) const { return (n + a.tile_rows - 1) / a.tile_rows; }
  // Tokens that some row of tile t sees (behind the last there may be anything), and units of its own ones: at least one, which leaves the row's
  // place in the partials in order.
  __device__ __forceinline__ int end(const CacheAttnArgs &a, int t) const { return a.tree ? len : max(0, len - n + min(n, (t + 1) * a.tile_rows)); }
  __device__ __forceinline__ int units(const CacheAttnArgs &a, int t) const { return max(1, (end(a, t) - a.shared_tokens + CA_BLK - 1) / CA_BLK); }
  __device__ __forceinline__ long long all_units(const CacheAttnArgs &a) const {
    long long sum = 0;
    for (int t = tiles(a) - 1; t >= 0; --t) sum += units(a, t);
    return sum * a.c.hkv;
  }
};

// What a CTA has to do: units [u, u_end) of the call, as segments.
template <bool PAGES> struct CaWalk {
  long long u, u_end, u_first;
  int upc;                                 // units per CTA
  long long prefix_units;
  int prefix_tiles, prefix_blocks, prefix_rows;
  int seq, tile;
  long long at;                            // where the units behind the prefix stand: those of (seq, tile) start here
  // the segment
  int phase, row0, rows, kvh, end;         // rows row0 .. row0 + rows - 1; keys from `end` on are nobody's
  int b0, b1, key0;                        // units of the item, whose first key is key0
  int follow;                              // CTAs that continue the item (of the segment that starts it)
  __device__ __forceinline__ void cut(long long item, int blocks) {
    b0 = (int)(u - item);
    b1 = b0 + (int)min((long long)(blocks - b0), u_end - u);
    follow = (int)(item + blocks - 1 - u_first) / upc;
    u += b1 - b0;
  }
  __device__ __forceinline__ bool next(const CacheAttnArgs &a) {
    if (u >= u_end) return false;
    if (PAGES) {
      const int blocks = prefix_blocks, item = (int)(u / blocks);
      phase = 1; row0 = item / a.c.hkv; rows = 1; kvh = item - row0 * a.c.hkv; seq = a.row_seq[row0]; key0 = 0; end = a.row_pos[row0];
      cut((long long)item * blocks, blocks);
      return true;
    }
    if (u < prefix_units) {
      const int item = (int)u / prefix_blocks;
      phase = 0; kvh = item / prefix_tiles;
      row0 = (item - kvh * prefix_tiles) * a.tile_rows; rows = min(a.tile_rows, prefix_rows - row0);
      end = a.shared_tokens; key0 = 0;
      cut(item * prefix_blocks, prefix_blocks);
      return true;
    }
    for (; seq < a.c.n_seqs; ++seq, tile = 0) {
      const CaSeq s(a, seq);
      for (const int tiles = s.tiles(a); tile < tiles; ++tile) {
        const int blocks = s.units(a, tile), sum = blocks * a.c.hkv;
        if (u < at + sum) {
          phase = 1; kvh = (int)(u - at) / blocks;
          row0 = s.q0 + tile * a.tile_rows; rows = min(a.tile_rows, s.n - tile * a.tile_rows);
          end = s.end(a, tile); key0 = a.shared_tokens;
          cut(at + kvh * blocks, blocks);
          return true;
        }
        at += sum;
      }
    }
    return false;
  }
};

template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(CA_THREADS, (CaShape<HD>::CTAS_PER_SM))
k_cache_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CacheAttnArgs a) {
  using Sh = CaShape<HD>;
  constexpr int STAGES = Sh::STAGES, KP = Sh::KP;
  extern __shared__ uint8_t ca_smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)ca_smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *q_s = smem, *k_s = q_s + Sh::Q_BYTES, *v_s = k_s + STAGES * Sh::STAGE;
  uint64_t *bars = (uint64_t *)(v_s + STAGES * Sh::STAGE);
  uint64_t *k_full = bars, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES;
  uint64_t *s_full = v_empty + STAGES, *p_full = s_full + 2, *o_done = p_full + 2, *q_full = o_done + 2, *o_free = q_full + 1;
  volatile uint64_t *masks = (volatile uint64_t *)(o_free + 1);            // [CA_MASKS] which keys of a unit there are
  uint32_t *tmem_base_p = (uint32_t *)(masks + CA_MASKS);
  volatile int *abort_flag = (volatile int *)(tmem_base_p + 1);
  __shared__ long long sh_sum[CA_THREADS / 32], sh_at;
  __shared__ int sh_seq, sh_partial, sh_status[2];

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, cta = blockIdx.x;
  unsigned long long *tr = trace_open();
  if (warp == 0) {
    if (lane < STAGES) { mbar_init(k_full + lane, 1); mbar_init(k_empty + lane, 1); mbar_init(v_full + lane, 1); mbar_init(v_empty + lane, 1); }
    else if (lane >= 8 && lane < 10) { mbar_init(s_full + lane - 8, 1); mbar_init(p_full + lane - 8, 4); mbar_init(o_done + lane - 8, 1); }
    else if (lane == 16) { mbar_init(q_full, 4); mbar_init(o_free, 4); *abort_flag = 0; }
    else if (lane == 17) { sh_partial = 0; sh_seq = 0; sh_at = 0; sh_status[0] = sh_status[1] = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_base_p)), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  trace_stamp(tr, TR_k_cache_attn);
  int *status = a.status ? a.status : sh_status;

  // ---- this CTA's units
  CaWalk<PAGES> w;
  long long total;
  if (PAGES) {
    w.prefix_blocks = max(1, (a.budget * a.c.page_tokens + CA_BLK - 1) / CA_BLK);
    total = (long long)a.rows * a.c.hkv * w.prefix_blocks;
    w.prefix_units = 0;
  } else {
    w.prefix_rows = min(max(a.q_start[a.c.n_seqs], 0), a.rows);
    w.prefix_tiles = (w.prefix_rows + a.tile_rows - 1) / a.tile_rows;
    w.prefix_blocks = (a.shared_tokens + CA_BLK - 1) / CA_BLK;
    w.prefix_units = (long long)w.prefix_tiles * w.prefix_blocks * a.c.hkv;
    long long sum = 0;
    for (int s = threadIdx.x; s < a.c.n_seqs; s += CA_THREADS) {
      const CaSeq q(a, s);
      sum += q.all_units(a);
      if (q.n && q.len - q.n + (a.tree ? 0 : 1) < a.shared_tokens) sh_partial = 1;       // a row that does not see the whole prefix
      if (cta == 0 && (q.q0 != a.q_start[s] || q.q0 + q.n != a.q_start[s + 1] || q.len != a.kv_len[s])) cache_bad_index(status);
    }
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh_sum[warp] = sum;
    __syncthreads();
    total = w.prefix_units;
    for (int i = 0; i < CA_THREADS / 32; ++i) total += sh_sum[i];
  }
  w.upc = (int)max(1ll, (total + a.n_ctas - 1) / a.n_ctas);
  w.u_first = (long long)cta * w.upc;
  w.u = min(w.u_first, total);
  w.u_end = min(w.u + w.upc, total);
  if (!PAGES && w.u < w.u_end) {
    // the sequence in which the units behind the prefix start for this CTA
    const long long goal = max(w.u, w.prefix_units);
    long long at = w.prefix_units;
    for (int s0 = 0; s0 < a.c.n_seqs && at <= goal; s0 += CA_THREADS) {
      const int s = s0 + threadIdx.x;
      const long long own = s < a.c.n_seqs ? CaSeq(a, s).all_units(a) : 0ll;
      long long sum = own;
      for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
      __syncthreads();
      if (lane == 31) sh_sum[warp] = sum;
      __syncthreads();
      long long before = at;
      for (int i = 0; i < CA_THREADS / 32; ++i) { if (i < warp) before += sh_sum[i]; at += sh_sum[i]; }
      before += sum - own;
      if (goal >= before && goal < before + own) { sh_seq = s; sh_at = before; }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_p;
  w.seq = sh_seq; w.tile = 0; w.at = sh_at;
  int gave_up = WAIT_none;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    const uint64_t pol = policy_evict_normal();
    const int sub = min(CA_BLK, a.c.page_tokens), n_sub = CA_BLK / sub;     // keys of one copy, copies of a unit
    int ks = 0, vs = 0, g = 0;
    uint32_t kph = 1, vph = 1;
    while (!gave_up && w.next(a)) {
      // lane l holds the page of part p0 + l of the item's keys, and the first of these keys in the sequence
      int p0 = -64, page = 0, token = 0;
      for (int blk = w.b0; blk < w.b1 && !gave_up; ++blk, ++g) {
        const int part = blk * n_sub;
        if (part < p0 || part + n_sub > p0 + 32) {
          p0 = part;
          const int first = (p0 + lane) * sub;             // key of the item
          page = -1;
          bool bad = false;
          if (PAGES) {
            const int e = first >> a.c.page_shift;
            const int *ids = a.ids + ((long long)w.row0 * a.c.hkv + w.kvh) * a.budget;
            token = 0;
            if (w.seq >= 0 && w.end >= 0) {
              if (!a.c.token_ok(w.seq, w.end)) bad = true;
              else if (e < a.budget) {
                const int id = ids[e], before = e ? ids[e - 1] : -1;
                if (id > before && id >= 0 && id <= w.end >> a.c.page_shift) {
                  token = (id << a.c.page_shift) + (first & (a.c.page_tokens - 1));
                  page = a.c.page(w.seq, id);
                  bad = page < 0;
                }
              }
            }
          } else {
            token = w.key0 + first;
            if (token < w.end) {
              page = a.c.page(w.phase ? w.seq : 0, token >> a.c.page_shift);
              bad = page < 0;
            }
          }
          if (bad) cache_bad_index(status);
        }
        // which of the unit's keys there are: of its parts with a page, those in front of the end
        uint32_t m0 = 0, m1 = 0;
        const int i = lane - (part - p0);
        if (i >= 0 && i < n_sub && page >= 0) {
          const int n = min(sub, max(0, (PAGES ? w.end + 1 : w.end) - token));
          const uint64_t m = (n >= 64 ? ~0ull : (1ull << n) - 1ull) << (i * sub);
          m0 = (uint32_t)m; m1 = (uint32_t)(m >> 32);
        }
        m0 = __reduce_or_sync(0xffffffffu, m0);
        m1 = __reduce_or_sync(0xffffffffu, m1);
        for (int which = 0; which < 2 && !gave_up; ++which) {
          int &st = which ? vs : ks;
          uint32_t &ph = which ? vph : kph;
          uint64_t *full = (which ? v_full : k_full) + st;
          uint8_t *dst = (which ? v_s : k_s) + st * Sh::STAGE;
          const CUtensorMap *map = which ? &map_v : &map_k;
          if (!mbar_wait_warp((which ? v_empty : k_empty) + st, ph, abort_flag)) { gave_up = WAIT_cache_kv_ring; break; }
          if (elect_one()) {
            if (!which) masks[g % CA_MASKS] = (uint64_t)m0 | (uint64_t)m1 << 32;
            mbar_expect_tx(full, (uint32_t)Sh::STAGE);
          }
          __syncwarp();
          for (int s = 0; s < n_sub; ++s) {
            // a part without a page is filled with zeros: its page number is past the last
            const int pg = __shfl_sync(0xffffffffu, page, part - p0 + s), tk = __shfl_sync(0xffffffffu, token, part - p0 + s) & (a.c.page_tokens - 1);
            if (elect_one()) {
              if (n_sub == 1) tma_load_5d(dst, map, full, 0, tk, 0, w.kvh, pg < 0 ? a.c.n_pages : pg, pol);
              else
                for (int kp = 0; kp < KP; ++kp) tma_load_5d(dst + kp * Sh::PANEL + s * sub * 128, map, full, 0, tk, kp, w.kvh, pg < 0 ? a.c.n_pages : pg, pol);
            }
            __syncwarp();
          }
          if (++st == STAGES) { st = 0; ph ^= 1u; }
        }
      }
    }
    // Until the last releases have arrived: one that came in after this CTA has left would land in the shared memory of the next.
#pragma unroll 1
    for (int i = 0; i < STAGES && !gave_up; ++i) {
      if (!mbar_wait_warp(k_empty + ks, kph, abort_flag) || !mbar_wait_warp(v_empty + vs, vph, abort_flag)) gave_up = WAIT_cache_last;
      if (++ks == STAGES) { ks = 0; kph ^= 1u; }
      if (++vs == STAGES) { vs = 0; vph ^= 1u; }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ matrix instructions: S of a unit, then O of the one before
    constexpr uint32_t id_s = (1u << 4) | CaType<T>::IDESC | ((uint32_t)(CA_BLK >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t id_o = (1u << 4) | CaType<T>::IDESC | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t qd = smem_desc(smem_u32(q_s)), kd = smem_desc(smem_u32(k_s)), vd = smem_desc_mn(smem_u32(v_s), Sh::PANEL);
    const uint32_t s_addr = tmem_base + HD;
    int ks = 0, vs = 0, g = 0, seg = 0;
    uint32_t kph = 0, vph = 0;
    // O of unit x (counted over the CTA's life), the first of its segment or not
    auto issue_o = [&](int x, bool first) {
      if (first && seg > 0 && !mbar_wait_warp(o_free, (uint32_t)(seg - 1) & 1u, abort_flag)) { gave_up = WAIT_cache_o; return; }
      if (!__all_sync(0xffffffffu, mbar_wait(v_full + vs, vph, abort_flag) && mbar_wait(p_full + (x & 1), (uint32_t)(x >> 1) & 1u, abort_flag))) { gave_up = WAIT_cache_p_v; return; }
      const uint64_t m = masks[x % CA_MASKS];
      if (m != ~0ull) {
        // values that are nobody's may be anything, and 0 times that not 0
        uint8_t *dst = v_s + vs * Sh::STAGE;
        for (int i = lane; i < CA_BLK * KP * 8; i += 32) {
          const int key = (i >> 3) & (CA_BLK - 1);
          if (!(m >> key & 1ull)) *reinterpret_cast<uint4 *>(dst + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
        __syncwarp();
      }
      tc_fence_after();
      if (elect_one()) {
        const uint64_t bd = vd + (uint64_t)((vs * Sh::STAGE) >> 4);
#pragma unroll
        for (int k = 0; k < CA_BLK / 16; ++k)                               // 16 keys: eight columns of P, two groups of eight rows of V
          mma_tmem_a(tmem_base, s_addr + (uint32_t)((x & 1) * CA_BLK + k * 8), bd + (uint64_t)(k * 128), id_o, (!first || k > 0) ? 1u : 0u);
        mma_commit(v_empty + vs);
        mma_commit(o_done + (x & 1));
      }
      __syncwarp();
      if (++vs == STAGES) { vs = 0; vph ^= 1u; }
    };
    while (!gave_up && w.next(a)) {
      const int n = w.b1 - w.b0;
      if (!mbar_wait_warp(q_full, (uint32_t)seg & 1u, abort_flag)) { gave_up = WAIT_cache_q; break; }
      for (int i = 0; i <= n && !gave_up; ++i) {
        if (i < n) {
          // (the buffer of S is free: O of the unit before last, which read P there, was issued before)
          if (!mbar_wait_warp(k_full + ks, kph, abort_flag)) { gave_up = WAIT_cache_k; break; }
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kp = 0; kp < KP; ++kp)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                mma_bf16(s_addr + (uint32_t)(((g + i) & 1) * CA_BLK), qd + (uint64_t)((kp * Sh::Q_PANEL + k * 32) >> 4),
                         kd + (uint64_t)((ks * Sh::STAGE + kp * Sh::PANEL + k * 32) >> 4), id_s, (kp > 0 || k > 0) ? 1u : 0u);
            mma_commit(k_empty + ks);
            mma_commit(s_full + ((g + i) & 1));
          }
          __syncwarp();
          if (++ks == STAGES) { ks = 0; kph ^= 1u; }
        }
        if (i > 0) issue_o(g + i - 1, i == 1);
      }
      g += n;
      ++seg;
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue: a row of the tile per thread
    const int quarter = warp & 3, e = quarter * 32 + lane;                  // TMEM lanes this warp may access; entry of the tile
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) {                       // one lane polls for the warp
      int v = 1;
      if (lane == 0 && (!ok || !mbar_wait(bar, parity, abort_flag))) v = 0;
      if (!__shfl_sync(0xffffffffu, v, 0) && ok) {
        ok = false;
        if (lane == 0) wait_expired(status, WAIT_cache_softmax, abort_flag, -1);
      }
    };
    const float scale = a.scale_log2;
    int g = 0;
    bool more = w.next(a);
    // the queries of the segment ahead, this warp's 32 rows of the tile
    auto load_q = [&]() {
      const int n = w.rows * a.group;
      if (quarter * 32 < n) {
        constexpr int V = HD / 8;
#pragma unroll 4
        for (int i = lane; i < 32 * V; i += 32) {
          const int row = quarter * 32 + i / V, vec = i % V;
          if (row < n) {
            const int r = row / a.group, h = w.kvh * a.group + row - r * a.group;
            const uint4 x = *reinterpret_cast<const uint4 *>((const T *)a.q + (long long)(w.row0 + r) * a.q_ld + (long long)h * HD + vec * 8);
            *reinterpret_cast<uint4 *>(q_s + (vec >> 3) * Sh::Q_PANEL + row * 128 + (((vec & 7) ^ (row & 7)) << 4)) = x;
          }
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    };
    if (more) load_q();
    while (more) {
      const int n_entries = w.rows * a.group, n = w.b1 - w.b0, b0 = w.b0, key0 = w.key0, kvh = w.kvh, phase = w.phase, follow = w.follow;
      const bool active = quarter * 32 < n_entries, mine = e < n_entries, starts = b0 == 0;
      const int r = w.row0 + e / a.group, h = kvh * a.group + e % a.group;
      // what the row sees: keys below vis, and key tail0 + j where bit j of the mask is set
      int vis = 0x7fffffff, tail0 = 0;
      unsigned long long mlo = 0ull, mhi = 0ull;
      const bool row_on = !PAGES || w.seq >= 0;
      if (!PAGES && mine && (phase || sh_partial)) {
        int s = w.seq;
        if (!phase) {                                                       // the sequence that has the row
          int lo = 0, hi = a.c.n_seqs;
          while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (a.q_start[m] <= r) lo = m; else hi = m; }
          s = lo;
        }
        const CaSeq q(a, s);
        tail0 = q.len - q.n;
        vis = a.tree ? tail0 : tail0 + (r - q.q0) + 1;
        if (a.tree) {
          const uint32_t *t = a.tree + (long long)r * 4;
          mlo = t[0] | (unsigned long long)t[1] << 32;
          mhi = t[2] | (unsigned long long)t[3] << 32;
        }
      }
      const bool tree = !PAGES && a.tree;
      float m_ref = -INFINITY, l = 0.f, l_true = 0.f;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int x = g + i, j0 = key0 + (b0 + i) * CA_BLK;
        wait(s_full + (x & 1), (uint32_t)(x >> 1) & 1u);
        // A wait is for a phase whose predecessor is known to be over: O of the unit before last, whose barrier this unit's O has too, is waited for here
        // (it was issued before S).
        if (x > 1) wait(o_done + (x & 1), (uint32_t)((x >> 1) - 1) & 1u);
        if (active) {
          tc_fence_after();
          const uint32_t s_col = lane_addr + (uint32_t)(HD + (x & 1) * CA_BLK);
          uint32_t s0[32], s1[32];
          tmem_ld32(s_col, s0);
          tmem_ld32(s_col + 32, s1);
          uint64_t vm = masks[x % CA_MASKS];
          if (!PAGES) {
            const int npre = min(64, max(0, vis - j0));
            unsigned long long m = npre >= 64 ? ~0ull : (1ull << npre) - 1ull;
            if (tree && npre < 64) {
              const int sh = j0 - tail0;                                    // node of key j0
              if (sh < 0) m |= sh > -64 ? mlo << (-sh) : 0ull;
              else if (sh < 64) m |= (mlo >> sh) | (sh ? mhi << (64 - sh) : 0ull);
              else m |= sh < 128 ? mhi >> (sh - 64) : 0ull;
            }
            vm &= m;
          }
          tmem_ld_wait();
          if (__any_sync(0xffffffffu, vm != ~0ull)) {
            const uint32_t v0 = (uint32_t)vm, v1 = (uint32_t)(vm >> 32);
#pragma unroll
            for (int c = 0; c < 32; ++c) {
              s0[c] = v0 >> c & 1u ? s0[c] : 0xff800000u;
              s1[c] = v1 >> c & 1u ? s1[c] : 0xff800000u;
            }
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            mx[0] = fmaxf(mx[0], __uint_as_float(s0[c])); mx[1] = fmaxf(mx[1], __uint_as_float(s0[c + 1]));
            mx[2] = fmaxf(mx[2], __uint_as_float(s1[c])); mx[3] = fmaxf(mx[3], __uint_as_float(s1[c + 1]));
          }
          const float bm = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
          const bool grow = mine && bm > m_ref + CaType<T>::RESCALE && m_ref != -INFINITY;
          if (__any_sync(0xffffffffu, grow)) {
            // the accumulator takes the new reference, behind the O of every earlier unit
            wait(o_done + ((x - 1) & 1), (uint32_t)((x - 1) >> 1) & 1u);
            tc_fence_after();
            const float corr = grow ? ex2(m_ref - bm) : 1.f;
#pragma unroll 1
            for (int c0 = 0; c0 < HD; c0 += 32) {
              uint32_t o[32];
              tmem_ld32(lane_addr + (uint32_t)c0, o);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * corr);
              tmem_st32(lane_addr + (uint32_t)c0, o);
            }
            if (grow) { l *= corr; l_true *= corr; m_ref = bm; }
          }
          if (m_ref == -INFINITY) m_ref = bm;
          const float nbase = (m_ref == -INFINITY ? 0.f : -m_ref) + CaType<T>::SHIFT;
          uint32_t p[32];
          float sum[2] = {0.f, 0.f}, sum_true[2] = {0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float p0 = ex2(fmaf(__uint_as_float(s0[c]), scale, nbase)), p1 = ex2(fmaf(__uint_as_float(s0[c + 1]), scale, nbase));
            const float p2 = ex2(fmaf(__uint_as_float(s1[c]), scale, nbase)), p3 = ex2(fmaf(__uint_as_float(s1[c + 1]), scale, nbase));
            p[c / 2] = pack2(p0, p1, T());
            p[16 + c / 2] = pack2(p2, p3, T());
            const float2 u = unpack2(p[c / 2], T()), v = unpack2(p[16 + c / 2], T());
            sum[0] += u.x + u.y; sum[1] += v.x + v.y;
            sum_true[0] += p0 + p1; sum_true[1] += p2 + p3;
          }
          l += sum[0] + sum[1];
          l_true += sum_true[0] + sum_true[1];
          tmem_st32(s_col, p);
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + (x & 1));
      }
      g += n;
      more = w.next(a);
      if (more) load_q();                                                   // (S of the last unit is done: nobody reads the queries any more)
      wait(o_done + ((g - 1) & 1), (uint32_t)((g - 1) >> 1) & 1u);
      if (active && ok) {
        tc_fence_after();
        const float m = m_ref == -INFINITY ? m_ref : m_ref - CaType<T>::SHIFT;
        const long long rh = (long long)r * a.heads + h;
        const bool final = starts && !follow && (PAGES || !a.shared_tokens);
        const long long at = starts ? (PAGES ? rh : (long long)phase * a.rows * a.heads + rh) : (long long)cta * 128 + e;
        float *po = (starts ? a.part_o : a.cont_o) + at * HD;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        T *out = (T *)a.out + (long long)r * a.out_ld + (long long)h * HD;
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          uint32_t o[32];
          tmem_ld32(lane_addr + (uint32_t)c0, o);
          tmem_ld_wait();
          if (!mine) continue;
          if (final) {
            if (row_on) {
              const float f = l > 0.f ? inv : 0.f;
#pragma unroll
              for (int c = 0; c < 32; c += 8) {
                uint32_t z[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) z[k] = pack2(__uint_as_float(o[c + 2 * k]) * f, __uint_as_float(o[c + 2 * k + 1]) * f, T());
                *reinterpret_cast<uint4 *>(out + c0 + c) = make_uint4(z[0], z[1], z[2], z[3]);
              }
            }
          } else {
#pragma unroll
            for (int c = 0; c < 32; c += 4) *reinterpret_cast<uint4 *>(po + c0 + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
          }
        }
        if (mine) {
          if (starts) {
            a.part_ml[at] = make_float4(m, l, l_true, pack_follow(e, final || !row_on ? CA_DONE : follow, cta + 1));
            if (final && row_on && a.lse) a.lse[rh] = l > 0.f ? (m + log2f(l_true)) * 0.6931471805599453f : -INFINITY;
          } else a.cont_ml[at] = make_float4(m, l, l_true, 0.f);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_free);
    }
  }
  if (gave_up && lane == 0) wait_expired(status, gave_up, abort_flag, -1);
  drain_if_aborted(abort_flag);
  pdl_trigger();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
  }
}

// The segments of a (row, head), from the first to the last: out = sum w O / sum w l with w = 2^(m - max m).  A thread takes eight columns.  PHASES: 1, or 2 where
// the shared pages have partials of their own.
template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(256)
k_cache_merge(const __grid_constant__ CacheAttnArgs a) {
  kernel_entry(TR_k_cache_merge);
  constexpr int V = HD / 8;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, rh = i / V;
  const int c0 = (int)(i % V) * 8, r = (int)(rh / a.heads);
  if (r >= a.rows || (!PAGES && r >= a.q_start[a.c.n_seqs])) return;
  float M = -INFINITY, L = 0.f, Lt = 0.f, acc[8] = {};
  const int first = PAGES || a.shared_tokens ? 0 : 1;
  for (int phase = first; phase < (PAGES ? 1 : 2); ++phase) {
    const long long at = (long long)phase * a.rows * a.heads + rh;
    float4 ml = a.part_ml[at];
    const int f = __float_as_int(ml.w), entry = f & 127, cta = f >> 18 & 0x3ff;
    int n = f >> 7 & 0x7ff;
    if (n == CA_DONE) return;
    n = min(n, a.n_ctas - cta);
    const float *po = a.part_o + at * HD;
    for (int k = 0;; ++k) {
      const float Mn = fmaxf(M, ml.x);
      if (ml.x != -INFINITY) {
        const float sc = ex2(M - Mn), w = ex2(ml.x - Mn);
        const float4 x = *reinterpret_cast<const float4 *>(po + c0), y = *reinterpret_cast<const float4 *>(po + c0 + 4);
        L = L * sc + ml.y * w; Lt = Lt * sc + ml.z * w;
        acc[0] = acc[0] * sc + x.x * w; acc[1] = acc[1] * sc + x.y * w; acc[2] = acc[2] * sc + x.z * w; acc[3] = acc[3] * sc + x.w * w;
        acc[4] = acc[4] * sc + y.x * w; acc[5] = acc[5] * sc + y.y * w; acc[6] = acc[6] * sc + y.z * w; acc[7] = acc[7] * sc + y.w * w;
        M = Mn;
      }
      if (k >= n) break;
      const long long c = (long long)(cta + k) * 128 + entry;
      ml = a.cont_ml[c];
      po = a.cont_o + c * HD;
    }
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] *= inv;
  *reinterpret_cast<uint4 *>((T *)a.out + r * a.out_ld + (rh - (long long)r * a.heads) * HD + c0) = pack8<T>(acc);
  if (a.lse && c0 == 0) a.lse[rh] = L > 0.f ? (M + log2f(Lt)) * 0.6931471805599453f : -INFINITY;
}
