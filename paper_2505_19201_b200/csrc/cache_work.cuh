// How the work of the attention over a paged cache is dealt out, and how its parts come together again.
//
// Work.  An item is a tile of query entries (entry = (row, query head of one KV-head group)), up to 128 or up to 4 by kernel, against a run of keys of one KV head, cut into
// units of 64 or 128 keys.  Shared pages: the rows of all sequences stand together, in full tiles, so that the prefix is read once for all of them (once per
// tile; see ca_shared).  A sequence's own tokens: its rows, tile by tile, in the launch for its number of entries.  Listed pages: one row.  The units of all items, one behind the other, are dealt out to
// the CTAs in equal contiguous ranges, by arithmetic on the lengths that each CTA does for itself (they are on the device), so long contexts
// with few rows fill the GPU and short ones do not leave a tail.  An item counts START units more than it has, for what starting and ending it costs.  A
// range is a few segments, each in one item.  A segment leaves (m, l, O) of its keys; k_cache_merge adds up the
// segments of a row, always in the same order.  The segment that starts an item has its place by row and head, a CTA's continuation
// of an item the CTA's own.
#pragma once
#include "attn_tc.cuh"
#include "cache_rows.cuh"

#define CA_RING 16                       // units' key masks, and segments, that are known at once: more than the stages and the buffers of S together

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
  int shared_tokens;                       // dense: keys [0, shared_tokens) are everybody's (see ca_shared)
  float scale_log2;
  float *part_o;                           // [phase][row][head][HD]: what the segment that starts an item leaves ...
  float4 *part_ml;                         // [phase][row][head]: its (m, l, l before rounding, what follows: see pack_follow)
  float *cont_o;                           // [CTA][128][HD], [CTA][128]: the segments that continue one
  float4 *cont_ml;
  int with_prefix, own_from, own_to;       // dense: what this launch takes, the shared keys or not, and the own keys of sequences with so many query entries to a KV head
  int n_ctas, cont_base, cont_slots;       // CTAs of this launch, where its continuations' slots start, and slots of all launches
  int early;                               // the launch in front is the other one of this call, of which this one needs nothing ...
  int let;                                 // ... and this one has the other behind it, which may begin where blocks of this one have left
  int look;                                // merge: most rows are one segment, and done
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

// The shared keys that are an item of their own, against the rows of all sequences.  Sequences whose own rows fill tiles read the prefix once per tile either way, and then it is one item
// with their own keys, whose parts need not be put together: 0.  (Seven sequences behind 4096 tokens, 16 heads over 8 of 256, with 128 rows each 89 us, and 113 with the prefix by itself;
// with 64 rows 61 and 64, but their last tiles are full, which at other lengths they are not; with 32 rows 46 and 40.)  From two tiles to a sequence on, on the average over the
// sequences, the tiles by sequence are at most half as many again as those of all rows together, however the rows are spread: one more for each sequence (31 tokens and a prompt of 2100 rows behind 4352, 32 heads over 8 of 128, 302 us, and 350 with the prefix by itself).  The rows counted are those there
// are, not those that a captured call has room for.
__device__ __forceinline__ int ca_shared(const CacheAttnArgs &a, int n_rows) { return (long long)n_rows * a.group >= 256ll * a.c.n_seqs ? 0 : a.shared_tokens; }
__device__ __forceinline__ int ca_rows(const CacheAttnArgs &a) { return min(max(a.q_start[a.c.n_seqs], 0), a.rows); }

// A sequence as the call gives it, held within the buffers whatever its numbers say.
struct CaSeq {
  int q0, n, len;                          // first row, rows, tokens
  CaSeq() = default;
  __device__ __forceinline__ CaSeq(const CacheAttnArgs &a, int s) {
    q0 = min(max(a.q_start[s], 0), a.rows);
    n = min(max(a.q_start[s + 1], q0), a.rows) - q0;
    len = min(max(a.kv_len[s], 0), a.c.pages_per_seq << a.c.page_shift);
  }
  __device__ __forceinline__ bool taken(const CacheAttnArgs &a) const { return n * a.group >= a.own_from && n * a.group <= a.own_to; }      // by this launch
  __device__ __forceinline__ int tiles(const CacheAttnArgs &a) const { return (n + a.tile_rows - 1) / a.tile_rows; }
  // Tokens that some row of tile t sees (behind the last there may be anything), and units of its own ones: at least one, which leaves the row's
  // place in the partials in order.
  __device__ __forceinline__ int end(const CacheAttnArgs &a, int t) const { return a.tree ? len : max(0, len - n + min(n, (t + 1) * a.tile_rows)); }
  template <int BLK> __device__ __forceinline__ int units(const CacheAttnArgs &a, int t, int shared) const { return max(1, (end(a, t) - shared + BLK - 1) / BLK); }
  template <int BLK, int START> __device__ __forceinline__ long long all_units(const CacheAttnArgs &a, int shared) const {
    long long sum = 0;
    for (int t = tiles(a) - 1; t >= 0; --t) sum += units<BLK>(a, t, shared) + START;
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
  int tail0, q0;                           // phase 1: the sequence's tokens in front of its rows', and the first of these
};

// The sequence that has row r.
__device__ __forceinline__ int ca_seq_of(const CacheAttnArgs &a, int r) {
  int lo = 0, hi = a.c.n_seqs;
  while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (a.q_start[m] <= r) lo = m; else hi = m; }
  return lo;
}

struct CaPlanShared { long long sum[32], at; CaSeq q; int seq, partial, longest, shared; };      // partial and longest start as 0

// a / b for a from 0 and b from 1 on: a division of 64-bit numbers takes several times that of 32-bit ones, and hardly a call has as many units.
__device__ __forceinline__ long long ca_div(long long a, int b) { return a >> 31 ? a / b : (long long)((int)a / b); }

// What a CTA has to do: units [u, u_end) of the call, as segments.  Every item is reached from the one before it by counting on; lengths are read once per sequence.
template <int BLK, int START, bool PAGES> struct CaWalk {
  long long u, u_end, u_first, item;       // item: the first unit of the item at hand, which has START + blocks
  int upc, blocks, tile, tiles, shared;
  int prefix_tiles, prefix_blocks, prefix_rows;
  CaSeq q;
  CaSeg s;

  __device__ __forceinline__ void at_row(const CacheAttnArgs &a, int row) {               // pages: the first KV head of a row
    s.row0 = row; s.kvh = 0;
    if (row < a.rows) { s.seq = a.row_seq[row]; s.end = a.row_pos[row]; }
  }
  __device__ __forceinline__ void at_tile(const CacheAttnArgs &a) {                       // own keys: the first KV head of a tile of sequence s.seq
    blocks = q.template units<BLK>(a, tile, shared);
    s.row0 = q.q0 + tile * a.tile_rows; s.rows = min(a.tile_rows, q.n - tile * a.tile_rows);
    s.end = q.end(a, tile); s.tail0 = q.len - q.n; s.q0 = q.q0; s.kvh = 0;
  }
  __device__ __forceinline__ void at_own(const CacheAttnArgs &a, int seq) {               // ... the first tile of this sequence
    s.phase = 1; s.seq = seq; s.key0 = shared;
    tile = 0;
    tiles = q.tiles(a);
    if (tiles) at_tile(a);
    else u = u_end;                                          // (none: lengths that changed under way)
  }
  // ... of the first sequence from this one on that this launch takes; by a whole warp, which looks at 32 sequences at a time (8 of 4096 slots with a row each: 33 us; one by one 65).
  __device__ __forceinline__ void at_seq(const CacheAttnArgs &a, int seq) {
    q.n = 0;
    for (; seq < a.c.n_seqs; seq += 32) {
      const int i = seq + (threadIdx.x & 31);
      CaSeq t;
      t.q0 = t.n = t.len = 0;
      if (i < a.c.n_seqs) t = CaSeq(a, i);
      const unsigned some = __ballot_sync(0xffffffffu, t.taken(a));
      if (some) {
        const int first = __ffs(some) - 1;
        seq += first;
        q.q0 = __shfl_sync(0xffffffffu, t.q0, first); q.n = __shfl_sync(0xffffffffu, t.n, first); q.len = __shfl_sync(0xffffffffu, t.len, first);
        break;
      }
    }
    at_own(a, seq);
  }
  __device__ __forceinline__ void at_prefix(const CacheAttnArgs &a) {                     // shared keys: a tile of KV head s.kvh
    s.row0 = tile * a.tile_rows; s.rows = min(a.tile_rows, prefix_rows - tile * a.tile_rows);
  }
  __device__ __forceinline__ void next_item(const CacheAttnArgs &a) {
    item += START + blocks;
    if (PAGES) {
      if (++s.kvh == a.c.hkv) at_row(a, s.row0 + 1);
    } else if (s.phase) {
      if (++s.kvh < a.c.hkv) return;
      if (++tile < tiles) at_tile(a);
      else at_seq(a, s.seq + 1);
    } else {
      if (++tile == prefix_tiles) { tile = 0; ++s.kvh; }
      if (s.kvh < a.c.hkv) at_prefix(a);
      else at_seq(a, 0);
    }
  }
  // The next segment, in s.
  __device__ __forceinline__ bool next(const CacheAttnArgs &a) {
    while (u < u_end) {
      if (u >= item + START + blocks) { next_item(a); continue; }
      // behind START units that stand for the item's start; nothing where the range ends among them
      s.b0 = max((int)(u - item) - START, 0);
      s.n = (int)min((long long)blocks, u_end - item - START) - s.b0;
      s.follow = (int)(item + START + blocks - 1 - u_first) / upc;
      u = min(u_end, item + START + blocks);
      if (s.n > 0) return true;
    }
    s.n = 0;
    return false;
  }

  // What this CTA has to do, from lengths that are on the device: by all threads of the block.
  __device__ __forceinline__ void plan(const CacheAttnArgs &a, CaPlanShared &sh, int *status) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, cta = blockIdx.x;
    long long total, prefix_units = 0;
    tile = tiles = shared = 0;
    s.key0 = s.seq = s.kvh = s.tail0 = s.q0 = 0;
    if (PAGES) {
      blocks = max(1, (a.budget * a.c.page_tokens + BLK - 1) / BLK);
      total = (long long)a.rows * a.c.hkv * (blocks + START);
      upc = (int)max(1ll, ca_div(total + a.n_ctas - 1, a.n_ctas));
    } else {
      prefix_rows = ca_rows(a);
      shared = ca_shared(a, prefix_rows);
      if (threadIdx.x == 0) sh.shared = shared;
      prefix_blocks = (shared + BLK - 1) / BLK;
      prefix_tiles = prefix_blocks && a.with_prefix ? (prefix_rows + a.tile_rows - 1) / a.tile_rows : 0;
      prefix_units = (long long)prefix_tiles * (prefix_blocks + START) * a.c.hkv;
      // units in front of each sequence's, a sequence per thread at a time; once around for most batches, twice where there are more sequences than threads
      long long own = 0, sum = 0;
      int longest = 0;
      CaSeq t;
      for (int i = threadIdx.x; i < a.c.n_seqs; i += blockDim.x) {
        t = CaSeq(a, i);
        own = t.taken(a) ? t.template all_units<BLK, START>(a, shared) : 0ll;
        sum += own;
        if (t.n && t.len - t.n + (a.tree ? 0 : 1) < shared) sh.partial = 1;       // a row that does not see the whole prefix
        if (t.n) longest = max(longest, t.len);
        if (cta == 0 && (t.q0 != a.q_start[i] || (i == 0 && t.q0) || t.q0 + t.n != a.q_start[i + 1] || t.len != a.kv_len[i])) cache_bad_index(status);
      }
      for (int o = 1; o < 32; o <<= 1) { const long long x = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += x; }
      longest = __reduce_max_sync(0xffffffffu, longest);
      if (lane == 31) { sh.sum[warp] = sum; if (longest) atomicMax(&sh.longest, longest); }
      __syncthreads();
      total = prefix_units;
      long long before = prefix_units + sum - own;
      for (int i = 0; i < warps; ++i) { if (i < warp) before += sh.sum[i]; total += sh.sum[i]; }
      // the sequence in which the units behind the prefix start for this CTA
      upc = (int)max(1ll, ca_div(total + a.n_ctas - 1, a.n_ctas));
      const long long goal = max(min((long long)cta * upc, total), prefix_units);
      if (a.c.n_seqs <= (int)blockDim.x) {
        if (goal >= before && goal < before + own) { sh.seq = threadIdx.x; sh.at = before; sh.q = t; }
      } else {
        long long next = prefix_units;
        for (int i0 = 0; i0 < a.c.n_seqs && next <= goal; i0 += blockDim.x) {
          const int i = i0 + threadIdx.x;
          if (i < a.c.n_seqs) t = CaSeq(a, i);
          own = i < a.c.n_seqs && t.taken(a) ? t.template all_units<BLK, START>(a, shared) : 0ll;
          sum = own;
          for (int o = 1; o < 32; o <<= 1) { const long long x = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += x; }
          __syncthreads();
          if (lane == 31) sh.sum[warp] = sum;
          __syncthreads();
          before = next + sum - own;
          for (int k = 0; k < warps; ++k) { if (k < warp) before += sh.sum[k]; next += sh.sum[k]; }
          if (goal >= before && goal < before + own) { sh.seq = i; sh.at = before; sh.q = t; }
        }
      }
      __syncthreads();
    }
    u_first = (long long)cta * upc;
    u = min(u_first, total);
    u_end = min(u + upc, total);
    if (u >= u_end) return;
    // ---- the item in which the range starts
    if (PAGES) {
      const int i = (int)ca_div(u, blocks + START), row = i / a.c.hkv;
      s.phase = 1; s.rows = 1;
      at_row(a, row);
      s.kvh = i - row * a.c.hkv;
      item = (long long)i * (blocks + START);
    } else if (u < prefix_units) {
      const int i = (int)u / (prefix_blocks + START);
      s.phase = 0; s.end = min(shared, sh.longest);                               // behind everybody's last token there may be anything
      blocks = prefix_blocks;
      s.kvh = i / prefix_tiles; tile = i - s.kvh * prefix_tiles;
      item = (long long)i * (prefix_blocks + START);
      at_prefix(a);
    } else {
      item = sh.at;
      q = sh.q;
      at_own(a, sh.seq);
      for (; tile < tiles; at_tile(a)) {                     // the tile, then the KV head
        const long long all = (long long)(blocks + START) * a.c.hkv;
        if (u < item + all) break;
        item += all;
        if (++tile == tiles) break;
      }
      s.kvh = (int)(u - item) / (blocks + START);
      item += (long long)s.kvh * (blocks + START);
    }
  }
};

// Whether a phase is over, without waiting.
__device__ __forceinline__ bool mbar_test(uint64_t *bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return done != 0;
}

// K (WHICH = 0) or V (1) of all units, by a warp of its own, with what goes with a unit and a segment for the others (WHICH = 0 alone).  Returns the wait that ran out.
struct CaRing { uint64_t *full, *empty, *seg_full; uint8_t *data; uint4 *masks; CaSeg *segs; const CUtensorMap *map; volatile int *abort_flag; int *status; };
template <int HD, int STAGES, int WHICH, int BLK, int START, bool PAGES>
__device__ __forceinline__ int ca_produce(const CacheAttnArgs &a, CaWalk<BLK, START, PAGES> &w, const CaRing &ring, int lane) {
  constexpr int KP = HD / 64, STAGE = BLK * HD * 2, PANEL = BLK * 128;
  const uint64_t pol = policy_evict_normal();
  const int sub = min(BLK, a.c.page_tokens), n_sub = BLK / sub;             // keys of one copy, copies of a unit
  int st = 0, g = 0, gave_up = WAIT_none;
  uint32_t ph = 1;
  // lane l holds the page of part p0 + l of the item's keys, and the first of these keys in the sequence; good for the items of one (seq, phase, end)
  int p0 = -64, page = 0, token = 0, of_seq = -1, of_phase = -1, of_end = -1;
  for (int n_seg = 0;; ++n_seg) {
    w.next(a);
    if (!WHICH) {
      if (elect_one()) {
        ring.segs[n_seg % CA_RING] = w.s;
        mbar_arrive(ring.seg_full + n_seg % CA_RING);
      }
      __syncwarp();
    }
    if (!w.s.n) break;
    const CaSeg &s = w.s;
    if (PAGES || s.seq != of_seq || s.phase != of_phase || s.end != of_end) { p0 = -64; of_seq = s.seq; of_phase = s.phase; of_end = s.end; }
    for (int blk = s.b0; blk < s.b0 + s.n; ++blk, ++g) {
      const int part = blk * n_sub;
      if (part < p0 || part + n_sub > p0 + 32) {
        p0 = part;
        const int first = (p0 + lane) * sub;                 // key of the item
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
        if (bad) cache_bad_index(ring.status);
      }
      uint4 m = make_uint4(0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu);
      if (!WHICH) {
        // which of the unit's keys there are: of its parts with a page, those in front of the end
        const int i = lane - (part - p0), k0 = i * sub, k1 = page >= 0 ? k0 + min(sub, max(0, (PAGES ? s.end + 1 : s.end) - token)) : k0;
        const bool on = i >= 0 && i < n_sub;
        if (__any_sync(0xffffffffu, on && k1 - k0 < sub)) {
          uint32_t x[4];
#pragma unroll
          for (int k = 0; k < BLK / 32; ++k) {
            const int lo = max(k0 - 32 * k, 0), hi = min(k1 - 32 * k, 32);
            x[k] = __reduce_or_sync(0xffffffffu, on && hi > lo ? (0xffffffffu >> (32 - (hi - lo))) << lo : 0u);
          }
          m = make_uint4(x[0], x[1], BLK > 64 ? x[2] : 0u, BLK > 64 ? x[3] : 0u);
        }
      }
      if (!mbar_wait_warp(ring.empty + st, ph, ring.abort_flag)) { gave_up = WAIT_cache_kv_ring; break; }
      if (elect_one()) {
        if (!WHICH) ring.masks[g % CA_RING] = m;
        mbar_expect_tx(ring.full + st, (uint32_t)STAGE);
      }
      __syncwarp();
      uint8_t *dst = ring.data + st * STAGE;
      for (int j = 0; j < n_sub; ++j) {
        // a part without a page is filled with zeros: its page number is past the last
        const int pg = __shfl_sync(0xffffffffu, page, part - p0 + j), tk = __shfl_sync(0xffffffffu, token, part - p0 + j) & (a.c.page_tokens - 1);
        if (elect_one()) {
          if (n_sub == 1) tma_load_5d(dst, ring.map, ring.full + st, 0, tk, 0, s.kvh, pg < 0 ? a.c.n_pages : pg, pol);
          else
            for (int kp = 0; kp < KP; ++kp) tma_load_5d(dst + kp * PANEL + j * sub * 128, ring.map, ring.full + st, 0, tk, kp, s.kvh, pg < 0 ? a.c.n_pages : pg, pol);
        }
        __syncwarp();
      }
      if (++st == STAGES) { st = 0; ph ^= 1u; }
    }
    if (gave_up) break;
  }
  // Until the last releases have arrived: one that came in after this CTA has left would land in the shared memory of the next.
#pragma unroll 1
  for (int i = 0; i < STAGES && !gave_up; ++i) {
    if (!mbar_wait_warp(ring.empty + st, ph, ring.abort_flag)) gave_up = WAIT_cache_last;
    if (++st == STAGES) { st = 0; ph ^= 1u; }
  }
  return gave_up;
}

// The segments of a (row, head), from the first to the last: out = sum w O / sum w l with w = 2^(m - max m).  Threads with four columns each do this together, and take
// four segments at a time, so that their loads are under way together.  Bound by the latency of those loads, one round behind another.  (Eight segments at a time: four trees of 61
// nodes 32.7 us as a whole in place of 29.5; eight columns a thread: 30.4, and seven prompts of 500 tokens, 256 wide, 163 in place of 159.)
// Where most rows are one segment, and done, a block looks over MERGE_LOOK of them first (look), and does not load the partial results that are not there.
#define MERGE_LOOK 32                    // of a block's first warp, a lane each
template <typename T, int HD, bool PAGES>
__device__ __forceinline__ void merge_row(const CacheAttnArgs &a, bool shared, long long rh, int r, int c0) {
  float M = -INFINITY, L = 0.f, Lt = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4 &ml, const float4 &x) {
    if (ml.x == -INFINITY) return;
    const float Mn = fmaxf(M, ml.x), sc = ex2(M - Mn), w = ex2(ml.x - Mn);
    L = L * sc + ml.y * w; Lt = Lt * sc + ml.z * w;
    acc.x = acc.x * sc + x.x * w; acc.y = acc.y * sc + x.y * w; acc.z = acc.z * sc + x.z * w; acc.w = acc.w * sc + x.w * w;
    M = Mn;
  };
  // what starts the row's items, shared and own
  const int first = PAGES || shared ? 0 : 1, last = PAGES ? 0 : 1;
  float4 ml[2], x[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const long long at = (long long)k * a.rows * a.heads + rh;
    const bool on = k >= first && k <= last;
    ml[k] = on ? a.part_ml[at] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    x[k] = on ? *reinterpret_cast<const float4 *>(a.part_o + at * HD + c0) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k < first || k > last) continue;
    const int f = __float_as_int(ml[k].w), entry = f & 127, cta = f >> 18 & 0x3ff;
    int n = f >> 7 & 0x7ff;
    if (n == CA_DONE) return;
    n = min(n, a.cont_slots - cta);
    add(ml[k], x[k]);
    auto some = [&](int j, auto count) {
      constexpr int N = decltype(count)::value;
      float4 cm[N], cx[N];
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const long long c = (long long)(cta + min(j + q, n - 1)) * 128 + entry;
        cm[q] = a.cont_ml[c];
        cx[q] = *reinterpret_cast<const float4 *>(a.cont_o + c * HD + c0);
      }
#pragma unroll
      for (int q = 0; q < N; ++q) if (j + q < n) add(cm[q], cx[q]);
    };
    int j = 0;
    for (; n - j > 2; j += 4) some(j, std::integral_constant<int, 4>());
    if (j < n) some(j, std::integral_constant<int, 2>());
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  *reinterpret_cast<uint2 *>((T *)a.out + r * a.out_ld + (rh - (long long)r * a.heads) * HD + c0) = make_uint2(pack2(acc.x * inv, acc.y * inv, T()), pack2(acc.z * inv, acc.w * inv, T()));
  if (a.lse && c0 == 0) a.lse[rh] = L > 0.f ? (M + log2f(Lt)) * 0.6931471805599453f : -INFINITY;
}
template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(256, 4)
k_cache_merge(const __grid_constant__ CacheAttnArgs a) {
  kernel_entry(TR_k_cache_merge);
  constexpr int V = HD / 4, PER = 256 / V;
  const int rows = PAGES ? a.rows : ca_rows(a), first = PAGES ? 0 : a.q_start[0];      // (rows in front of the first sequence are nobody's, and have no parts)
  const bool shared = !PAGES && ca_shared(a, rows) > 0;
  const int c0 = (int)(threadIdx.x % V) * 4;
  if (!a.look) {
    const long long rh = (long long)blockIdx.x * PER + threadIdx.x / V;
    const int r = (int)ca_div(rh, a.heads);
    if (r >= first && r < rows) merge_row<T, HD, PAGES>(a, shared, rh, r, c0);
    return;
  }
  __shared__ int list[MERGE_LOOK], n_list;
  const long long base = (long long)blockIdx.x * MERGE_LOOK;
  const int t = threadIdx.x;
  if (t < 32) {
    const long long rh = base + t;
    const bool open = t < MERGE_LOOK && ca_div(rh, a.heads) < rows && ca_div(rh, a.heads) >= first && (__float_as_int(a.part_ml[(PAGES ? 0ll : (long long)a.rows * a.heads) + rh].w) >> 7 & 0x7ff) != CA_DONE;
    const unsigned b = __ballot_sync(0xffffffffu, open);
    if (open) list[__popc(b & ((1u << t) - 1u))] = t;
    if (t == 0) n_list = __popc(b);
  }
  __syncthreads();
  const int n = n_list;
  for (int j = t / V; j < n; j += PER) {
    const long long rh = base + list[j];
    merge_row<T, HD, PAGES>(a, shared, rh, (int)ca_div(rh, a.heads), c0);
  }
}
