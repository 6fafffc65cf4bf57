// Attention over a paged cache that a program holds itself, on the tcgen05 tensor cores: a ragged batch whose sequences may begin with the
// same pages (dream_cache_attn), and rows that read listed pages (dream_cache_attn_pages).
//
// Work.  An item is up to 128 query entries (entry = (row, query head of one KV-head group)) against a run of keys of one KV head, cut into
// units of 64 keys.  Shared pages: the rows of all sequences stand together, in tiles of 128 entries, so that the prefix is read once for all of them (once per
// tile).  A sequence's own tokens: its rows, tile by tile.  Listed pages: one row.  The units of all items, one behind the other, are dealt out to
// the CTAs in equal contiguous ranges, by arithmetic on the lengths that each CTA does for itself (they are on the device), so long contexts
// with few rows fill the GPU and short ones do not leave a tail.  An item counts CA_START units more than it has, for what starting and ending it costs.  A
// range is a few segments, each in one item.  A segment leaves (m, l, O) of its keys; k_cache_merge adds up the
// segments of a row, always in the same order.  The segment that starts an item has its place by row and head, a CTA's continuation
// of an item the CTA's own.
//
// A segment.  S = Q K^T (128 x 64, fp32 in TMEM, two to four buffers), softmax by eight warps of 16 rows each, the four lanes of a quad to a row (and to the
// one eight further on): one pass with a running reference m that follows the
// row's maximum only when that has outgrown it (the accumulator is then rescaled, seldom), P = 2^(s - m) rounded to the cache's type into the columns
// its scores came from, O += P V with P as the TMEM operand.  l sums the rounded P, so that the weights add up to 1 whatever their rounding, which
// then moves the result by at most half a step of sum w |v - out|; the log-sum-exp has a sum of its own, of P as it was.  K and V come by TMA in two rings that
// run on from segment to segment, so that the next one's keys are under way while one ends.  The producer alone works out what the segments are, ahead of
// everybody else, and leaves them in a ring in shared memory.
// Warps: 0 TMA and segments, 1 S, Q and TMEM, 2 O, 3 nothing, 4..11 softmax and epilogue.  Two CTAs share an SM's registers: 80 for each thread, of which
// the first four warps leave the others a part.
#pragma once
#include "attn_tc.cuh"
#include "cache_rows.cuh"

#define CA_THREADS 384
#define CA_WARPS (CA_THREADS / 32)
#define CA_BLK 64                        // keys of a unit
#define CA_RING 16                       // units' key masks, and segments, that are known at once: more than the stages and the buffers of S together
#define CA_START 1                       // units that starting and ending an item is worth

template <int HD> struct CaShape {
  static constexpr int KP = HD / 64;                                   // 64-column panels of a row
  static constexpr int STAGES = HD == 64 ? 5 : 2;                      // units of K (and of V) in shared memory
  static constexpr int S_BUFS = HD == 64 ? 3 : HD == 128 ? 2 : 4;      // what the TMEM columns hold beside O
  static constexpr int TMEM_COLS = HD + S_BUFS * CA_BLK <= 256 ? 256 : 512;
  static constexpr int CTAS_PER_SM = HD == 256 ? 1 : 2;                // one walks its keys while the other starts or ends a segment
  static constexpr int Q_BYTES = 128 * HD * 2, Q_PANEL = 128 * 128;
  static constexpr int STAGE = CA_BLK * HD * 2, PANEL = CA_BLK * 128;
  static constexpr bool SPLIT = CTAS_PER_SM == 2;                      // registers are moved between the warps: 4 x 32 x 64 + 8 x 32 x 88 = 384 x 80
  static constexpr size_t SMEM = 1024 + Q_BYTES + 2 * STAGES * STAGE + 1536;
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
  int q_small;                             // query rows that the smaller of the two copies of Q takes
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
// 16 lanes x 32 columns: lane 4 i + j of the warp puts r[2 c] into column 4 c + j of TMEM lane i, r[2 c + 1] into that of lane i + 8.
__device__ __forceinline__ void tmem_st16x32(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
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
    for (int t = tiles(a) - 1; t >= 0; --t) sum += units(a, t) + CA_START;
    return sum * a.c.hkv;
  }
};

// A segment, as the producer leaves it for the others.
struct CaSeg {
  int row0, rows, kvh, seq;                // rows row0 .. row0 + rows - 1 against KV head kvh (phase 1: of sequence seq)
  int phase;                               // 0: shared keys; 1: the rows' own
  int end;                                 // keys from here on are nobody's (pages: the row's position)
  int b0, n, key0;                         // units b0 .. b0 + n - 1 of the item, whose first key is key0; n = 0: there are no more segments
  int follow;                              // CTAs that continue the item (of the segment that starts it)
};

// What a CTA has to do: units [u, u_end) of the call, as segments.
template <bool PAGES> struct CaWalk {
  long long u, u_end, u_first;
  int upc;                                 // units per CTA
  long long prefix_units;
  int prefix_tiles, prefix_blocks, prefix_rows;
  int seq, tile;
  long long at;                            // where the units behind the prefix stand: those of (seq, tile) start here
  // The part of this CTA in an item of so many blocks: behind CA_START units that stand for its start.  False where the range ends in front of the first.
  __device__ __forceinline__ bool cut(CaSeg &s, long long item, int blocks) {
    const int off = (int)(u - item) - CA_START;
    s.b0 = max(off, 0);
    const int b1 = (int)min((long long)blocks, u_end - item - CA_START);
    s.n = b1 - s.b0;
    s.follow = (int)(item + CA_START + blocks - 1 - u_first) / upc;
    u = min(u_end, item + CA_START + blocks);
    return s.n > 0;
  }
  __device__ __forceinline__ bool next(const CacheAttnArgs &a, CaSeg &s) {
    if (PAGES) {
      while (u < u_end) {
        const int blocks = prefix_blocks, item = (int)(u / (blocks + CA_START));
        s.phase = 1; s.row0 = item / a.c.hkv; s.rows = 1; s.kvh = item - s.row0 * a.c.hkv; s.seq = a.row_seq[s.row0]; s.key0 = 0; s.end = a.row_pos[s.row0];
        if (cut(s, (long long)item * (blocks + CA_START), blocks)) return true;
      }
      return false;
    }
    while (u < min(u_end, prefix_units)) {
      const int item = (int)u / (prefix_blocks + CA_START);
      s.phase = 0; s.seq = 0; s.kvh = item / prefix_tiles;
      s.row0 = (item - s.kvh * prefix_tiles) * a.tile_rows; s.rows = min(a.tile_rows, prefix_rows - s.row0);
      s.end = a.shared_tokens; s.key0 = 0;
      if (cut(s, (long long)item * (prefix_blocks + CA_START), prefix_blocks)) return true;
    }
    for (; u < u_end && seq < a.c.n_seqs; ++seq, tile = 0) {
      const CaSeq q(a, seq);
      for (const int tiles = q.tiles(a); tile < tiles; ++tile) {
        const int blocks = q.units(a, tile), each = blocks + CA_START;
        const long long sum = (long long)each * a.c.hkv;
        while (u < u_end && u < at + sum) {
          s.phase = 1; s.seq = seq; s.kvh = (int)(u - at) / each;
          s.row0 = q.q0 + tile * a.tile_rows; s.rows = min(a.tile_rows, q.n - tile * a.tile_rows);
          s.end = q.end(a, tile); s.key0 = a.shared_tokens;
          if (cut(s, at + (long long)s.kvh * each, blocks)) return true;
        }
        if (u >= u_end) return false;
        at += sum;
      }
    }
    return false;
  }
};

template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(CA_THREADS, (CaShape<HD>::CTAS_PER_SM))
k_cache_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q,
             const __grid_constant__ CUtensorMap map_q_small, const __grid_constant__ CacheAttnArgs a) {
  using Sh = CaShape<HD>;
  constexpr int STAGES = Sh::STAGES, KP = Sh::KP, SB = Sh::S_BUFS;
  extern __shared__ uint8_t ca_smem_raw[];
  uint8_t *smem = (uint8_t *)(((uintptr_t)ca_smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t *q_s = smem, *k_s = q_s + Sh::Q_BYTES, *v_s = k_s + STAGES * Sh::STAGE;
  uint64_t *bars = (uint64_t *)(v_s + STAGES * Sh::STAGE);
  uint64_t *k_full = bars, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES;
  uint64_t *s_full = v_empty + STAGES, *p_full = s_full + SB, *o_done = p_full + SB, *q_full = o_done + SB, *o_free = q_full + 1, *seg_full = o_free + 1;
  volatile uint64_t *masks = (volatile uint64_t *)(seg_full + CA_RING);    // [CA_RING] which keys of a unit there are
  CaSeg *segs = (CaSeg *)(masks + CA_RING);                                // [CA_RING]
  uint32_t *tmem_base_p = (uint32_t *)(segs + CA_RING);
  volatile int *abort_flag = (volatile int *)(tmem_base_p + 1);
  __shared__ long long sh_sum[CA_WARPS], sh_at;
  __shared__ int sh_seq, sh_partial, sh_status[2];

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, cta = blockIdx.x;
  unsigned long long *tr = trace_open();
  if (warp == 0) {
    if (lane < STAGES) { mbar_init(k_full + lane, 1); mbar_init(k_empty + lane, 1); mbar_init(v_full + lane, 1); mbar_init(v_empty + lane, 1); }
    else if (lane >= 8 && lane < 8 + SB) { mbar_init(s_full + lane - 8, 1); mbar_init(p_full + lane - 8, 8); mbar_init(o_done + lane - 8, 1); }
    else if (lane >= 16) mbar_init(seg_full + lane - 16, 1);
    if (lane == 12) { mbar_init(q_full, 1); mbar_init(o_free, 8); *abort_flag = 0; }
    else if (lane == 13) { sh_partial = 0; sh_seq = 0; sh_at = 0; sh_status[0] = sh_status[1] = 0; }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 3 && lane == 0) {
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
  static_assert(CA_RING > STAGES + SB, "what the producer leaves is read until a unit's P is done");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  trace_stamp(tr, TR_k_cache_attn);
  int *status = a.status ? a.status : sh_status;

  // ---- this CTA's units
  CaWalk<PAGES> w;
  long long total;
  w.seq = w.tile = 0;
  w.at = 0;
  if (PAGES) {
    w.prefix_blocks = max(1, (a.budget * a.c.page_tokens + CA_BLK - 1) / CA_BLK);
    total = (long long)a.rows * a.c.hkv * (w.prefix_blocks + CA_START);
    w.upc = (int)max(1ll, (total + a.n_ctas - 1) / a.n_ctas);
  } else {
    w.prefix_rows = min(max(a.q_start[a.c.n_seqs], 0), a.rows);
    w.prefix_blocks = (a.shared_tokens + CA_BLK - 1) / CA_BLK;
    w.prefix_tiles = w.prefix_blocks ? (w.prefix_rows + a.tile_rows - 1) / a.tile_rows : 0;
    w.prefix_units = (long long)w.prefix_tiles * (w.prefix_blocks + CA_START) * a.c.hkv;
    // units in front of each sequence's, a sequence per thread at a time; once around for most batches, twice where there are more sequences than threads
    const bool once = a.c.n_seqs <= CA_THREADS;
    long long own = 0, sum = 0;
    for (int s = threadIdx.x; s < a.c.n_seqs; s += CA_THREADS) {
      const CaSeq q(a, s);
      own = q.all_units(a);
      sum += own;
      if (q.n && q.len - q.n + (a.tree ? 0 : 1) < a.shared_tokens) sh_partial = 1;       // a row that does not see the whole prefix
      if (cta == 0 && (q.q0 != a.q_start[s] || q.q0 + q.n != a.q_start[s + 1] || q.len != a.kv_len[s])) cache_bad_index(status);
    }
    for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
    if (lane == 31) sh_sum[warp] = sum;
    __syncthreads();
    total = w.prefix_units;
    long long before = w.prefix_units + sum - own;
    for (int i = 0; i < CA_WARPS; ++i) { if (i < warp) before += sh_sum[i]; total += sh_sum[i]; }
    w.upc = (int)max(1ll, (total + a.n_ctas - 1) / a.n_ctas);
    // the sequence in which the units behind the prefix start for this CTA
    const long long goal = max(min((long long)cta * w.upc, total), w.prefix_units);
    if (once) {
      if (goal >= before && goal < before + own) { sh_seq = threadIdx.x; sh_at = before; }
    } else {
      long long at = w.prefix_units;
      for (int s0 = 0; s0 < a.c.n_seqs && at <= goal; s0 += CA_THREADS) {
        const int s = s0 + threadIdx.x;
        own = s < a.c.n_seqs ? CaSeq(a, s).all_units(a) : 0ll;
        sum = own;
        for (int o = 1; o < 32; o <<= 1) { const long long t = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += t; }
        __syncthreads();
        if (lane == 31) sh_sum[warp] = sum;
        __syncthreads();
        before = at + sum - own;
        for (int i = 0; i < CA_WARPS; ++i) { if (i < warp) before += sh_sum[i]; at += sh_sum[i]; }
        if (goal >= before && goal < before + own) { sh_seq = s; sh_at = before; }
      }
    }
    __syncthreads();
    w.seq = sh_seq; w.at = sh_at;
  }
  w.u_first = (long long)cta * w.upc;
  w.u = min(w.u_first, total);
  w.u_end = min(w.u + w.upc, total);
  const uint32_t tmem_base = *tmem_base_p;
  int gave_up = WAIT_none;
  // Units of segment number i, once the producer has left it; 0: there is none, or a wait ran out.
  auto segment = [&](int i, int where) {
    if (!mbar_wait_warp(seg_full + i % CA_RING, (uint32_t)(i / CA_RING) & 1u, abort_flag)) { gave_up = where; return 0; }
    return segs[i % CA_RING].n;
  };

  if (Sh::SPLIT) {
    if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
  }
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    const uint64_t pol = policy_evict_normal();
    const int sub = min(CA_BLK, a.c.page_tokens), n_sub = CA_BLK / sub;     // keys of one copy, copies of a unit
    int ks = 0, vs = 0, g = 0, n_seg = 0;
    uint32_t kph = 1, vph = 1;
    for (;; ++n_seg) {
      CaSeg s;
      if (!w.next(a, s)) s.n = 0;
      if (elect_one()) {
        segs[n_seg % CA_RING] = s;
        mbar_arrive(seg_full + n_seg % CA_RING);
      }
      __syncwarp();
      if (!s.n) break;
      // lane l holds the page of part p0 + l of the item's keys, and the first of these keys in the sequence
      int p0 = -64, page = 0, token = 0;
      for (int blk = s.b0; blk < s.b0 + s.n && !gave_up; ++blk, ++g) {
        const int part = blk * n_sub;
        if (part < p0 || part + n_sub > p0 + 32) {
          p0 = part;
          const int first = (p0 + lane) * sub;             // key of the item
          page = -1;
          token = 0;
          bool bad = false;
          if (PAGES) {
            const int e = first >> a.c.page_shift;
            const int *ids = a.ids + ((long long)s.row0 * a.c.hkv + s.kvh) * a.budget;
            if (s.seq >= 0 && s.end >= 0) {
              if (!a.c.token_ok(s.seq, s.end)) bad = true;
              else if (e < a.budget) {
                const int id = ids[e], before = e ? ids[e - 1] : -1;
                if (id > before && id >= 0 && id <= s.end >> a.c.page_shift) {
                  token = (id << a.c.page_shift) + (first & (a.c.page_tokens - 1));
                  page = a.c.page(s.seq, id);
                  bad = page < 0;
                }
              }
            }
          } else {
            token = s.key0 + first;
            if (token < s.end) {
              page = a.c.page(s.seq, token >> a.c.page_shift);
              bad = page < 0;
            }
          }
          if (bad) cache_bad_index(status);
        }
        // which of the unit's keys there are: of its parts with a page, those in front of the end
        uint32_t m0 = 0, m1 = 0;
        const int i = lane - (part - p0);
        if (i >= 0 && i < n_sub && page >= 0) {
          const int n = min(sub, max(0, (PAGES ? s.end + 1 : s.end) - token));
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
            if (!which) masks[g % CA_RING] = (uint64_t)m0 | (uint64_t)m1 << 32;
            mbar_expect_tx(full, (uint32_t)Sh::STAGE);
          }
          __syncwarp();
          for (int j = 0; j < n_sub; ++j) {
            // a part without a page is filled with zeros: its page number is past the last
            const int pg = __shfl_sync(0xffffffffu, page, part - p0 + j), tk = __shfl_sync(0xffffffffu, token, part - p0 + j) & (a.c.page_tokens - 1);
            if (elect_one()) {
              if (n_sub == 1) tma_load_5d(dst, map, full, 0, tk, 0, s.kvh, pg < 0 ? a.c.n_pages : pg, pol);
              else
                for (int kp = 0; kp < KP; ++kp) tma_load_5d(dst + kp * Sh::PANEL + j * sub * 128, map, full, 0, tk, kp, s.kvh, pg < 0 ? a.c.n_pages : pg, pol);
            }
            __syncwarp();
          }
          if (++st == STAGES) { st = 0; ph ^= 1u; }
        }
      }
      if (gave_up) break;
    }
    // Until the last releases have arrived: one that came in after this CTA has left would land in the shared memory of the next.
#pragma unroll 1
    for (int i = 0; i < STAGES && !gave_up; ++i) {
      if (!mbar_wait_warp(k_empty + ks, kph, abort_flag) || !mbar_wait_warp(v_empty + vs, vph, abort_flag)) gave_up = WAIT_cache_last;
      if (++ks == STAGES) { ks = 0; kph ^= 1u; }
      if (++vs == STAGES) { vs = 0; vph ^= 1u; }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ queries, and S = Q K^T: both operands K-major, N = 64
    constexpr uint32_t idesc = (1u << 4) | CaType<T>::IDESC | ((uint32_t)(CA_BLK >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
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
              mma_bf16(s_addr + (uint32_t)(sb * CA_BLK), qd + (uint64_t)((kp * Sh::Q_PANEL + k * 32) >> 4),
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
        const uint64_t m = masks[g % CA_RING];
        if (m != ~0ull) {
          // values that are nobody's may be anything, and 0 times that not 0
          uint8_t *dst = v_s + vs * Sh::STAGE;
#pragma unroll 1
          for (int j = lane; j < CA_BLK * KP * 8; j += 32)
            if (!(m >> ((j >> 3) & (CA_BLK - 1)) & 1ull)) *reinterpret_cast<uint4 *>(dst + j * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
          __syncwarp();
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t bd = vd + (uint64_t)((vs * Sh::STAGE) >> 4);
#pragma unroll
          for (int k = 0; k < CA_BLK / 16; ++k)                             // 16 keys: eight columns of P, two groups of eight rows of V
            mma_tmem_a(tmem_base, p_addr + (uint32_t)(sb * CA_BLK + k * 8), bd + (uint64_t)(k * 128), idesc, (i > 0 || k > 0) ? 1u : 0u);
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
    // ------------------------------------------------------------------ softmax and epilogue: warps 4..7 and 8..11 each take 16 lanes of a quarter; a
    // lane has 16 of a unit's 64 keys for two rows of the tile, e[0] and e[1] = e[0] + 8
    const int base = (warp & 3) * 32 + (warp >= 8 ? 16 : 0), quad = lane >> 2, ql = lane & 3;
    const uint32_t lane_addr = tmem_base + ((uint32_t)base << 16);
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
    const bool tree = !PAGES && a.tree;
    int g = 0, sb = 0;
    uint32_t sph = 0;
    for (int seg = 0, n; (n = segment(seg, WAIT_cache_softmax)) > 0; ++seg) {
      const CaSeg &s = segs[seg % CA_RING];              // read where it is needed: registers are short
      const int n_entries = s.rows * a.group;
      const bool active = base < n_entries, mine[2] = {base + quad < n_entries, base + quad + 8 < n_entries};
      // a row sees the keys below vis (of the item's first, units counted from the segment's first), and in a tree its own ones as the mask has them
      int vis[2] = {0x7fffffff, 0x7fffffff};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (!PAGES && mine[k] && (s.phase || sh_partial)) {
          const int r = s.row0 + (base + quad + 8 * k) / a.group;
          int sq = s.seq;
          if (!s.phase) {                                                   // the sequence that has the row
            int lo = 0, hi = a.c.n_seqs;
            while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (a.q_start[m] <= r) lo = m; else hi = m; }
            sq = lo;
          }
          const CaSeq q(a, sq);
          vis[k] = q.len - q.n + (tree ? 0 : r - q.q0 + 1) - (s.key0 + s.b0 * CA_BLK);
        }
      }
      float m_ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, l_true[2] = {0.f, 0.f};      // l: this lane's share of the sums
#pragma unroll 1
      for (int i = 0; i < n; ++i, ++g) {
        wait(s_full + sb, sph);
        if (active) {
          tc_fence_after();
          const uint32_t s_col = lane_addr + (uint32_t)(HD + sb * CA_BLK);
          uint32_t sr[32];                                                  // sr[4 c + 2 k + j]: row k, key 8 c + 2 ql + j
          tmem_ld16x64(s_col, sr);
          const uint64_t um = masks[g % CA_RING];
          const bool all = um == ~0ull && vis[0] - i * CA_BLK >= CA_BLK && vis[1] - i * CA_BLK >= CA_BLK;
          tmem_ld_wait();
          if (!__all_sync(0xffffffffu, all)) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int left = vis[k] - i * CA_BLK, npre = min(64, max(0, left));
              unsigned long long m = npre >= 64 ? ~0ull : (1ull << npre) - 1ull;
              if (tree && npre < 64 && mine[k]) {
                const uint32_t *t = a.tree + (long long)(s.row0 + (base + quad + 8 * k) / a.group) * 4;
                const unsigned long long mlo = t[0] | (unsigned long long)t[1] << 32, mhi = t[2] | (unsigned long long)t[3] << 32;
                const int sh = -left;                                       // node of the unit's first key
                if (sh < 0) m |= sh > -64 ? mlo << (-sh) : 0ull;
                else if (sh < 64) m |= (mlo >> sh) | (sh ? mhi << (64 - sh) : 0ull);
                else m |= sh < 128 ? mhi >> (sh - 64) : 0ull;
              }
              m = (m & um) >> (2 * ql);
              const uint32_t v0 = (uint32_t)m, v1 = (uint32_t)(m >> 32);
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const uint32_t v = c < 4 ? v0 >> (8 * c) : v1 >> (8 * c - 32);
                sr[4 * c + 2 * k] = v & 1u ? sr[4 * c + 2 * k] : 0xff800000u;
                sr[4 * c + 2 * k + 1] = v & 2u ? sr[4 * c + 2 * k + 1] : 0xff800000u;
              }
            }
          }
          float bm[2];
          bool grow[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float x = -INFINITY, y = -INFINITY;
#pragma unroll
            for (int c = 0; c < 8; ++c) { x = fmaxf(x, __uint_as_float(sr[4 * c + 2 * k])); y = fmaxf(y, __uint_as_float(sr[4 * c + 2 * k + 1])); }
            x = fmaxf(x, y);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            bm[k] = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2)) * scale;
            grow[k] = mine[k] && bm[k] > m_ref[k] + CaType<T>::RESCALE && m_ref[k] != -INFINITY;
          }
          if (__any_sync(0xffffffffu, grow[0] || grow[1])) {
            // the accumulator takes the new reference, behind the O of every earlier unit
            wait(o_done + (g - 1) % SB, (uint32_t)((g - 1) / SB) & 1u);
            tc_fence_after();
            const float corr0 = grow[0] ? ex2(m_ref[0] - bm[0]) : 1.f, corr1 = grow[1] ? ex2(m_ref[1] - bm[1]) : 1.f;
#pragma unroll 1
            for (int c0 = 0; c0 < HD; c0 += 64) {
              uint32_t o[32];
              tmem_ld16x64(lane_addr + (uint32_t)c0, o);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * (c & 2 ? corr1 : corr0));
              tmem_st16x64(lane_addr + (uint32_t)c0, o);
            }
            tmem_st_wait();
            if (grow[0]) { l[0] *= corr0; l_true[0] *= corr0; m_ref[0] = bm[0]; }
            if (grow[1]) { l[1] *= corr1; l_true[1] *= corr1; m_ref[1] = bm[1]; }
          }
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (m_ref[k] == -INFINITY) m_ref[k] = bm[k];
            const float nbase = (m_ref[k] == -INFINITY ? 0.f : -m_ref[k]) + CaType<T>::SHIFT;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float p0 = ex2(fmaf(__uint_as_float(sr[4 * c + 2 * k]), scale, nbase)), p1 = ex2(fmaf(__uint_as_float(sr[4 * c + 2 * k + 1]), scale, nbase));
              p[2 * c + k] = pack2(p0, p1, T());
              const float2 f = unpack2(p[2 * c + k], T());
              l[k] += f.x + f.y;
              l_true[k] += p0 + p1;
            }
          }
          tmem_st16x32(s_col, p);
          tmem_st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + sb);
        if (++sb == SB) { sb = 0; sph ^= 1u; }
      }
      // ---- epilogue
      const bool starts = s.b0 == 0, final = starts && !s.follow && (PAGES || !a.shared_tokens), row_on = !PAGES || s.seq >= 0;
      float inv[2];
      long long at[2];
      int r[2], h[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
        l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
        l_true[k] += __shfl_xor_sync(0xffffffffu, l_true[k], 1);
        l_true[k] += __shfl_xor_sync(0xffffffffu, l_true[k], 2);
        inv[k] = l[k] > 0.f ? 1.f / l[k] : 0.f;
        const int e = base + quad + 8 * k;
        r[k] = s.row0 + e / a.group;
        h[k] = s.kvh * a.group + e % a.group;
        const long long rh = (long long)r[k] * a.heads + h[k];
        at[k] = starts ? (PAGES ? rh : (long long)s.phase * a.rows * a.heads + rh) : (long long)cta * 128 + e;
        if (mine[k] && ql == 0) {
          const float m = m_ref[k] == -INFINITY ? m_ref[k] : m_ref[k] - CaType<T>::SHIFT;
          if (starts) {
            a.part_ml[at[k]] = make_float4(m, l[k], l_true[k], pack_follow(e, final || !row_on ? CA_DONE : s.follow, cta + 1));
            if (final && row_on && a.lse) a.lse[rh] = l[k] > 0.f ? (m + log2f(l_true[k])) * 0.6931471805599453f : -INFINITY;
          } else a.cont_ml[at[k]] = make_float4(m, l[k], l_true[k], 0.f);
        }
      }
      wait(o_done + (g - 1) % SB, (uint32_t)((g - 1) / SB) & 1u);
      if (active && ok) {
        tc_fence_after();
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 64) {
          uint32_t o[32];                                                   // o[4 c + 2 k + j]: row k, column c0 + 8 c + 2 ql + j
          tmem_ld16x64(lane_addr + (uint32_t)c0, o);
          tmem_ld_wait();
          if (final) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              T *out = (T *)a.out + (long long)r[k] * a.out_ld + (long long)h[k] * HD + c0;
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                uint32_t z[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) z[c] = pack2(__uint_as_float(o[16 * b + 4 * c + 2 * k]) * inv[k], __uint_as_float(o[16 * b + 4 * c + 2 * k + 1]) * inv[k], T());
                quad_transpose(z, lane);                                    // a lane now has eight columns that stand side by side
                if (mine[k] && row_on) *reinterpret_cast<uint4 *>(out + 32 * b + 8 * ql) = make_uint4(z[0], z[1], z[2], z[3]);
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              if (!mine[k]) continue;
              float *po = (starts ? a.part_o : a.cont_o) + at[k] * HD + c0 + 2 * ql;
#pragma unroll
              for (int c = 0; c < 8; ++c) *reinterpret_cast<uint2 *>(po + 8 * c) = make_uint2(o[4 * c + 2 * k], o[4 * c + 2 * k + 1]);
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
  pdl_trigger();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Sh::TMEM_COLS) : "memory");
  }
}

// The segments of a (row, head), from the first to the last: out = sum w O / sum w l with w = 2^(m - max m).  A thread takes eight columns, and of the segments four
// at a time, so that their loads are under way together.
template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(256)
k_cache_merge(const __grid_constant__ CacheAttnArgs a) {
  kernel_entry(TR_k_cache_merge);
  constexpr int V = HD / 8;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, rh = i / V;
  const int c0 = (int)(i % V) * 8, r = (int)(rh / a.heads);
  if (r >= a.rows || (!PAGES && r >= a.q_start[a.c.n_seqs])) return;
  float M = -INFINITY, L = 0.f, Lt = 0.f, acc[8] = {};
  auto add = [&](const float4 &ml, const float4 &x, const float4 &y) {
    if (ml.x == -INFINITY) return;
    const float Mn = fmaxf(M, ml.x), sc = ex2(M - Mn), w = ex2(ml.x - Mn);
    L = L * sc + ml.y * w; Lt = Lt * sc + ml.z * w;
    acc[0] = acc[0] * sc + x.x * w; acc[1] = acc[1] * sc + x.y * w; acc[2] = acc[2] * sc + x.z * w; acc[3] = acc[3] * sc + x.w * w;
    acc[4] = acc[4] * sc + y.x * w; acc[5] = acc[5] * sc + y.y * w; acc[6] = acc[6] * sc + y.z * w; acc[7] = acc[7] * sc + y.w * w;
    M = Mn;
  };
  // what starts the row's items, shared and own
  const int first = PAGES || a.shared_tokens ? 0 : 1, last = PAGES ? 0 : 1;
  float4 ml[2], x[2], y[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const long long at = (long long)k * a.rows * a.heads + rh;
    const bool on = k >= first && k <= last;
    ml[k] = on ? a.part_ml[at] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    x[k] = on ? *reinterpret_cast<const float4 *>(a.part_o + at * HD + c0) : make_float4(0.f, 0.f, 0.f, 0.f);
    y[k] = on ? *reinterpret_cast<const float4 *>(a.part_o + at * HD + c0 + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k < first || k > last) continue;
    const int f = __float_as_int(ml[k].w), entry = f & 127, cta = f >> 18 & 0x3ff;
    int n = f >> 7 & 0x7ff;
    if (n == CA_DONE) return;
    n = min(n, a.n_ctas - cta);
    add(ml[k], x[k], y[k]);
    for (int j = 0; j < n; j += 4) {
      float4 cm[4], cx[4], cy[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long c = (long long)(cta + min(j + q, n - 1)) * 128 + entry;
        cm[q] = a.cont_ml[c];
        cx[q] = *reinterpret_cast<const float4 *>(a.cont_o + c * HD + c0);
        cy[q] = *reinterpret_cast<const float4 *>(a.cont_o + c * HD + c0 + 4);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) if (j + q < n) add(cm[q], cx[q], cy[q]);
    }
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] *= inv;
  *reinterpret_cast<uint4 *>((T *)a.out + r * a.out_ld + (rh - (long long)r * a.heads) * HD + c0) = pack8<T>(acc);
  if (a.lse && c0 == 0) a.lse[rh] = L > 0.f ? (M + log2f(Lt)) * 0.6931471805599453f : -INFINITY;
}
