// Attention over a paged cache that a program holds itself.
#pragma once
#include "cache_rows.cuh"

struct CacheAttnArgs {
  CacheView c;
  const void *q;
  long long q_ld, out_ld;
  void *out;
  float *lse;
  const int *q_start, *kv_len;             // dense: rows by sequence
  const uint32_t *tree;                    // dense: [rows][4], or null
  const int *row_seq, *row_pos, *ids;      // pages
  int budget, rows, heads, group;
  float scale_log2;
  int *status;
};

// The simplest form: a block per row and query head, a warp per token in turn, softmax with a running maximum.
template <typename T, int HD, bool PAGES>
__global__ void __launch_bounds__(128)
k_cache_attn(const __grid_constant__ CacheAttnArgs a) {
  kernel_entry(TR_k_cache_attn);
  constexpr int E = HD / 32;
  const int r = blockIdx.x, h = blockIdx.y, kvh = h / a.group, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int seq, n, vis, tail0 = 0;
  if (PAGES) {
    seq = a.row_seq[r];
    if (seq < 0) return;
    vis = a.row_pos[r] + 1;
    if (vis < 1) vis = 0;
    else if (!a.c.token_ok(seq, vis - 1)) { if (threadIdx.x == 0) cache_bad_index(a.status); vis = 0; }
    n = a.budget * a.c.page_tokens;
  } else {
    int lo = 0, hi = a.c.n_seqs;            // the sequence whose rows hold r
    if (r >= a.q_start[hi]) return;
    while (hi - lo > 1) { const int m = (lo + hi) >> 1; if (a.q_start[m] <= r) lo = m; else hi = m; }
    seq = lo;
    const int T_ = a.q_start[seq + 1] - a.q_start[seq], given = a.kv_len[seq], len = min(max(given, 0), a.c.pages_per_seq << a.c.page_shift);
    if (given != len && threadIdx.x == 0) cache_bad_index(a.status);
    tail0 = len - T_;
    vis = a.tree ? tail0 : tail0 + (r - a.q_start[seq]) + 1;
    n = len;
  }
  __shared__ float sm[4], sl[4], so[4][HD];
  float q[E], o[E], m = -INFINITY, l = 0.f;
  const T *qp = (const T *)a.q + r * a.q_ld + (long long)h * HD;
#pragma unroll
  for (int i = 0; i < E; ++i) { q[i] = to_f(qp[lane + 32 * i]) * a.scale_log2; o[i] = 0.f; }
  for (int j = warp; j < n; j += 4) {
    int tok = j;
    if (PAGES) {
      const int *ids = a.ids + ((long long)r * a.c.hkv + kvh) * a.budget, e = j >> a.c.page_shift, id = ids[e];
      if (id < 0 || (e && id <= ids[e - 1])) continue;
      tok = (id << a.c.page_shift) + (j & (a.c.page_tokens - 1));
      if (id > (vis - 1) >> a.c.page_shift) continue;
    }
    if (tok >= vis) {
      const int b = tok - tail0;
      if (PAGES || !a.tree || b < 0 || b >= 128 || !(a.tree[(long long)r * 4 + b / 32] >> (b % 32) & 1u)) continue;
    }
    const int page = a.c.page(seq, tok >> a.c.page_shift);
    if (page < 0) { if (lane == 0) cache_bad_index(a.status); continue; }
    const long long at = a.c.at(page, kvh, tok & (a.c.page_tokens - 1));
    const T *k = (const T *)a.c.k + at, *v = (const T *)a.c.v + at;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += q[i] * to_f(k[lane + 32 * i]);
    s = warp_sum(s);
    const float mn = fmaxf(m, s), f = ex2(m - mn), p = ex2(s - mn);
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = o[i] * f + p * to_f(v[lane + 32 * i]);
    m = mn;
  }
#pragma unroll
  for (int i = 0; i < E; ++i) so[warp][lane + 32 * i] = o[i];
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
  __syncthreads();
  float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3])), L = 0.f, w[4];
  for (int i = 0; i < 4; ++i) { w[i] = sm[i] == -INFINITY ? 0.f : ex2(sm[i] - M); L += w[i] * sl[i]; }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  T *out = (T *)a.out + r * a.out_ld + (long long)h * HD;
  for (int d = threadIdx.x; d < HD; d += 128) out[d] = from_f<T>((w[0] * so[0][d] + w[1] * so[1][d] + w[2] * so[2][d] + w[3] * so[3][d]) * inv);
  if (a.lse && threadIdx.x == 0) a.lse[(long long)r * a.heads + h] = L > 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}
