// Entry points on a paged cache that a program holds itself (dream.h): checks on the host, then launches.  Part of dream_api.cu.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>
#include <climits>

#include "cache_attn.cuh"
#include "cache_few.cuh"
#include "cache_rows.cuh"

#define CACHE_MAX_ROWS (1 << 20)
#define CACHE_MAX_SEQS 4096
#define CACHE_MAX_BUDGET 4096
#define CACHE_MAX_SMS 160
#define CACHE_MAX_SELECT 32768             // pages of a sequence that dream_cache_select chooses from

// The view of a cache, or what is wrong with it.
static dream_status cache_view(const char *who, const dream_cache *c, CacheView *v) {
  if (!c) return fail(nullptr, DREAM_E_ARG, "%s: null cache", who);
  if (c->dtype != DREAM_BF16 && c->dtype != DREAM_F16) return fail(nullptr, DREAM_E_UNSUPPORTED, "%s: the cache's dtype must be DREAM_BF16 or DREAM_F16", who);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return fail(nullptr, DREAM_E_UNSUPPORTED, "%s: head_dim must be 64, 128 or 256", who);
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
    return fail(nullptr, DREAM_E_UNSUPPORTED, "%s: page_tokens must be a power of two in 16..256", who);
  if (!c->k || !c->v || !c->page_table) return fail(nullptr, DREAM_E_ARG, "%s: null k, v or page_table", who);
  if (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->bounds) & 15) return fail(nullptr, DREAM_E_ARG, "%s: k, v and bounds must be 16-byte aligned", who);
  if ((uintptr_t)c->page_table & 3) return fail(nullptr, DREAM_E_ARG, "%s: page_table is not aligned to its elements", who);
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_seqs < 1 || c->pages_per_seq < 1) return fail(nullptr, DREAM_E_ARG, "%s: n_pages, n_kv_heads, n_seqs and pages_per_seq must be positive", who);
  if (c->n_seqs > CACHE_MAX_SEQS) return fail(nullptr, DREAM_E_CAPACITY, "%s: n_seqs above %d", who, CACHE_MAX_SEQS);
  if (c->n_kv_heads > 1024) return fail(nullptr, DREAM_E_CAPACITY, "%s: n_kv_heads above 1024", who);
  if (c->pages_per_seq > (1 << 30) / c->page_tokens) return fail(nullptr, DREAM_E_CAPACITY, "%s: a sequence of more than 2^30 tokens", who);
  if (c->n_seqs > 1 && c->table_stride < c->pages_per_seq) return fail(nullptr, DREAM_E_ARG, "%s: rows of the page table overlap", who);
  // tokens of head_dim elements each in three directions, none of which may step into what the ones below it hold
  long long stride[3] = {c->token_stride, c->head_stride, c->page_stride}, count[3] = {c->page_tokens, c->n_kv_heads, c->n_pages};
  for (int i = 0; i < 3; ++i) {
    if (count[i] == 1) stride[i] = 0;                    // never stepped along
    else if (stride[i] < 1 || stride[i] % 8 || stride[i] >= 1LL << 38) return fail(nullptr, DREAM_E_ARG, "%s: strides must be positive multiples of 8 elements", who);
  }
  for (int i = 1; i < 3; ++i)
    for (int j = i; j > 0 && stride[j] < stride[j - 1]; --j) {
      long long t = stride[j]; stride[j] = stride[j - 1]; stride[j - 1] = t;
      t = count[j]; count[j] = count[j - 1]; count[j - 1] = t;
    }
  long long room = c->head_dim;
  for (int i = 0; i < 3; ++i) {
    if (count[i] == 1) continue;
    if (stride[i] < room) return fail(nullptr, DREAM_E_ARG, "%s: the strides make tokens overlap", who);
    room = stride[i] * (count[i] - 1) + room;
  }
  v->k = c->k; v->v = c->v; v->bounds = c->bounds; v->page_table = c->page_table;
  v->page_stride = c->n_pages > 1 ? c->page_stride : room; v->head_stride = c->n_kv_heads > 1 ? c->head_stride : c->head_dim;
  v->token_stride = c->token_stride; v->table_stride = c->table_stride;
  v->n_pages = c->n_pages; v->page_tokens = c->page_tokens; v->hkv = c->n_kv_heads; v->n_seqs = c->n_seqs; v->pages_per_seq = c->pages_per_seq;
  v->page_shift = 0;
  while (1 << v->page_shift < c->page_tokens) ++v->page_shift;
  return DREAM_OK;
}
static dream_status cache_heads(const char *who, const dream_cache *c, int rows, int n_heads) {
  if (rows < 1) return fail(nullptr, DREAM_E_ARG, "%s: rows = %d must be positive", who, rows);
  if (rows > CACHE_MAX_ROWS) return fail(nullptr, DREAM_E_CAPACITY, "%s: rows = %d above %d", who, rows, CACHE_MAX_ROWS);
  if (n_heads < 1 || n_heads % c->n_kv_heads) return fail(nullptr, DREAM_E_ARG, "%s: n_heads = %d is no multiple of n_kv_heads = %d", who, n_heads, c->n_kv_heads);
  if (n_heads / c->n_kv_heads > 128) return fail(nullptr, DREAM_E_UNSUPPORTED, "%s: more than 128 query heads per KV head", who);
  return DREAM_OK;
}
// A matrix of rows of heads x head_dim elements.
static dream_status cache_rows(const char *who, const char *name, const void *p, long long ld, long long width) {
  if (!p) return fail(nullptr, DREAM_E_ARG, "%s: %s is required", who, name);
  if ((uintptr_t)p & 15) return fail(nullptr, DREAM_E_ARG, "%s: %s must be 16-byte aligned", who, name);
  if (ld < width || ld % 8 || ld >= 1LL << 38) return fail(nullptr, DREAM_E_ARG, "%s: %s has rows of %lld elements, %lld apart (a multiple of 8, at least the row)", who, name, width, ld);
  return DREAM_OK;
}
static dream_status cache_ints(const char *who, const char *name, const void *p, bool needed) {
  if (!p && needed) return fail(nullptr, DREAM_E_ARG, "%s: %s is required", who, name);
  if ((uintptr_t)p & 3) return fail(nullptr, DREAM_E_ARG, "%s: %s is not aligned to its elements", who, name);
  return DREAM_OK;
}
static dream_status cache_workspace(const char *who, const void *p, size_t have, size_t need) {
  if (!p && need) return fail(nullptr, DREAM_E_ARG, "%s: workspace is required", who);
  if ((uintptr_t)p & 255) return fail(nullptr, DREAM_E_ARG, "%s: workspace must be 256-byte aligned", who);
  if (have < need) return fail(nullptr, DREAM_E_NOMEM, "%s: workspace needs %zu bytes, got %zu", who, need, have);
  return DREAM_OK;
}
template <typename... A>
static const char *cache_launch(void (*kernel)(A...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const A &...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = pdl_on() ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e == cudaSuccess) return nullptr;
  cudaGetLastError();
  return cudaGetErrorString(e);
}

extern "C" dream_status dream_rope_table(float *table, int32_t n_pos, int32_t rot_dim, float theta, void *cuda_stream) {
  if (!table || (uintptr_t)table & 15) return fail(nullptr, DREAM_E_ARG, "dream_rope_table: table must be 16-byte aligned device memory");
  if (n_pos < 1 || rot_dim < 16 || rot_dim > 256 || rot_dim % 16) return fail(nullptr, DREAM_E_ARG, "dream_rope_table: n_pos must be positive and rot_dim a multiple of 16 in 16..256");
  if (!(theta > 0.f) || isinf(theta)) return fail(nullptr, DREAM_E_ARG, "dream_rope_table: theta must be finite and above zero");
  k_rope_table<<<n_pos, 128, 0, (cudaStream_t)cuda_stream>>>((float2 *)table, rot_dim, theta);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? fail(nullptr, DREAM_E_CUDA, "dream_rope_table: %s", cudaGetErrorString(e)) : DREAM_OK;
}

extern "C" dream_status dream_cache_append(const dream_cache *cache, const void *q, int64_t q_ld, int32_t n_heads, const void *k_new, int64_t k_ld,
                                           const void *v_new, int64_t v_ld, int32_t rows, const int32_t *row_seq, const int32_t *slots,
                                           const int32_t *positions, const float *rope, int32_t n_pos, int32_t rot_dim, int32_t interleaved,
                                           void *q_out, int64_t q_out_ld, int32_t *status, void *cuda_stream) {
  static const char who[] = "dream_cache_append";
  CacheAppendArgs a = {};
  dream_status s = cache_view(who, cache, &a.c);
  if (s) return s;
  const int hd = cache->head_dim;
  if (!q != !q_out || (n_heads == 0) != !q) return fail(nullptr, DREAM_E_ARG, "%s: q, q_out and n_heads go together", who);
  s = cache_heads(who, cache, rows, q ? n_heads : cache->n_kv_heads);
  if (!s && q) s = cache_rows(who, "q", q, q_ld, (long long)n_heads * hd);
  if (!s && q) s = cache_rows(who, "q_out", q_out, q_out_ld, (long long)n_heads * hd);
  if (!s) s = cache_rows(who, "k_new", k_new, k_ld, (long long)cache->n_kv_heads * hd);
  if (!s) s = cache_rows(who, "v_new", v_new, v_ld, (long long)cache->n_kv_heads * hd);
  if (!s) s = cache_ints(who, "row_seq", row_seq, true);
  if (!s) s = cache_ints(who, "slots", slots, true);
  if (!s) s = cache_ints(who, "positions", positions, false);
  if (!s) s = cache_ints(who, "status", status, false);
  if (s) return s;
  if (rope) {
    if ((uintptr_t)rope & 15) return fail(nullptr, DREAM_E_ARG, "%s: rope must be 16-byte aligned", who);
    if (n_pos < 1) return fail(nullptr, DREAM_E_ARG, "%s: n_pos must be positive", who);
    if (rot_dim < 16 || rot_dim > hd || rot_dim % 16) return fail(nullptr, DREAM_E_ARG, "%s: rot_dim must be a multiple of 16 up to head_dim", who);
  }
  if (q && rows_collide(q, q_ld, q_out, q_out_ld, DREAM_BF16, rows, n_heads * hd)) return fail(nullptr, DREAM_E_ARG, "%s: q_out overlaps q without being q", who);
  a.q = q; a.q_ld = q_ld; a.k_new = k_new; a.k_ld = k_ld; a.v_new = v_new; a.v_ld = v_ld; a.q_out = q_out; a.q_out_ld = q_out_ld;
  a.row_seq = row_seq; a.slots = slots; a.positions = positions; a.rope = (const float2 *)rope; a.rows = rows; a.heads = q ? n_heads : 0; a.hd = hd;
  a.n_pos = n_pos; a.rot = rope ? rot_dim : 0; a.interleaved = interleaved != 0; a.status = status;
  // A thread takes one unit of one head where there are few rows, so that many share the latency; else that unit of several heads, whose rotary factors and place it looks up
  // once.  (32 + 2 x 8 heads of 128, with bounds, one head or several: 512 rows 9.5 or 9.2 us, 1024 rows 13.9 or 10.9, 3200 rows 35.1 or 21.5.)
  const int per = CACHE_THREADS / (hd / 16), n_heads_all = a.heads + 2 * a.c.hkv;
  const bool deep = (long long)rows * n_heads_all * (hd / 16) >= 2LL * CACHE_THREADS * 148 * 4;
  a.head_lanes = deep ? 1 : per;
  a.block_rows = per / a.head_lanes;
  a.head_blocks = (n_heads_all + a.head_lanes * (deep ? APPEND_HEADS : 1) - 1) / (a.head_lanes * (deep ? APPEND_HEADS : 1));
  a.bound_rows = 0;
  int chunk_rows = a.block_rows;
  a.bound_blocks = 0;
  if (a.c.bounds) {
    // A block looks over so many rows for full pages (a power of two): few where there are few rows, all of which may fill one at once.
    for (a.bound_rows = 1; a.bound_rows < 32 && (long long)rows * a.c.hkv >= 2LL * a.bound_rows * 148 * 4;) a.bound_rows *= 2;
    if (a.bound_rows > chunk_rows) chunk_rows = a.bound_rows;
    a.bound_blocks = chunk_rows / a.bound_rows * a.c.hkv;
  }
  a.chunk_rows = chunk_rows;
  a.chunk_blocks = a.bound_blocks + chunk_rows / a.block_rows * a.head_blocks;
  const long long blocks = (long long)((rows + chunk_rows - 1) / chunk_rows) * a.chunk_blocks;
  if (blocks > 0x7fffffffLL) return fail(nullptr, DREAM_E_CAPACITY, "%s: %d rows of %d heads in one call", who, rows, a.heads);
  void (*kernel)(CacheAppendArgs) = cache->dtype == DREAM_BF16 ? (deep ? k_cache_append<bf16, APPEND_HEADS> : k_cache_append<bf16, 1>)
                                                               : (deep ? k_cache_append<f16, APPEND_HEADS> : k_cache_append<f16, 1>);
  const char *why = cache_launch(kernel, dim3((unsigned)blocks), CACHE_THREADS, 0, (cudaStream_t)cuda_stream, a);
  return why ? fail(nullptr, DREAM_E_CUDA, "%s: %s", who, why) : DREAM_OK;
}

// The parts of the selection's workspace; how many bytes they are.
static size_t cache_select_room(const CacheView &v, int rows, void *workspace, CacheSelectArgs *a) {
  // Blocks of the scores for each (row, KV head): as many as fill the GPU, and no more than there are pages for
  const long long n = (long long)rows * v.hkv;
  const int most = (v.pages_per_seq + SCORE_PAGES - 1) / SCORE_PAGES;
  const long long share = 148 * SCORE_BLOCKS / n;
  const int blocks = share < 1 ? 1 : share < most ? (int)share : most;
  const size_t scores = ((size_t)n * v.pages_per_seq * sizeof(float) + 255) / 256 * 256;
  if (a) { a->scores = (float *)workspace; a->off = (float *)((char *)workspace + scores); a->score_blocks = blocks; }
  return scores + ((size_t)n * blocks * sizeof(float) + 255) / 256 * 256;
}

extern "C" dream_status dream_cache_select_bytes(const dream_cache *cache, int32_t rows, size_t *bytes) {
  CacheView v;
  dream_status s = cache_view("dream_cache_select_bytes", cache, &v);
  if (!s) s = cache_heads("dream_cache_select_bytes", cache, rows, cache->n_kv_heads);
  if (s) return s;
  if (!bytes) return fail(nullptr, DREAM_E_ARG, "dream_cache_select_bytes: null argument");
  *bytes = cache_select_room(v, rows, nullptr, nullptr);
  return DREAM_OK;
}

template <typename T, int HD>
static const char *cache_select_run(const CacheSelectArgs &a, int rows, cudaStream_t stream) {
  const char *why = nullptr;
  size_t smem = 0;
  if (a.c.pages_per_seq > a.budget) {
    why = cache_launch(k_cache_scores<T, HD>, dim3(rows * a.c.hkv, a.score_blocks), CACHE_THREADS, 0, stream, a);
    smem = (size_t)a.c.pages_per_seq * sizeof(uint32_t);      // of as many pages as a sequence may have
  }
  if (!why && smem > 32 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(k_cache_select<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, CACHE_MAX_SELECT * (int)sizeof(uint32_t));
    if (e != cudaSuccess) { cudaGetLastError(); why = cudaGetErrorString(e); }
  }
  return why ? why : cache_launch(k_cache_select<T, HD>, dim3(rows * a.c.hkv), SELECT_THREADS, smem, stream, a);
}

extern "C" dream_status dream_cache_select(const dream_cache *cache, const void *q, int64_t q_ld, int32_t n_heads, int32_t rows, const int32_t *row_seq,
                                           const int32_t *row_pos, int32_t budget, int32_t keep_first, int32_t keep_last, int32_t *ids,
                                           void *workspace, size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  static const char who[] = "dream_cache_select";
  CacheSelectArgs a = {};
  size_t need = 0;
  dream_status s = cache_view(who, cache, &a.c);
  if (!s) s = cache_heads(who, cache, rows, n_heads);
  if (!s) s = cache_rows(who, "q", q, q_ld, (long long)n_heads * cache->head_dim);
  if (!s) s = cache_ints(who, "row_seq", row_seq, true);
  if (!s) s = cache_ints(who, "row_pos", row_pos, true);
  if (!s) s = cache_ints(who, "ids", ids, true);
  if (!s) s = cache_ints(who, "status", status, false);
  if (s) return s;
  if (!cache->bounds) return fail(nullptr, DREAM_E_ARG, "%s: the cache has no bounds", who);
  if (keep_first < 0 || keep_last < 1 || keep_first > CACHE_MAX_BUDGET || keep_last > CACHE_MAX_BUDGET || budget < keep_first + keep_last)
    return fail(nullptr, DREAM_E_ARG, "%s: budget = %d must hold keep_first = %d >= 0 and keep_last = %d >= 1", who, budget, keep_first, keep_last);
  if (budget > CACHE_MAX_BUDGET) return fail(nullptr, DREAM_E_CAPACITY, "%s: budget above %d", who, CACHE_MAX_BUDGET);
  if (cache->pages_per_seq > CACHE_MAX_SELECT) return fail(nullptr, DREAM_E_CAPACITY, "%s: pages_per_seq above %d", who, CACHE_MAX_SELECT);
  if ((long long)rows * cache->n_kv_heads > 0x7fffffffLL) return fail(nullptr, DREAM_E_CAPACITY, "%s: %d rows in one call", who, rows);
  s = dream_cache_select_bytes(cache, rows, &need);
  if (!s) s = cache_workspace(who, workspace, workspace_bytes, need);
  if (s) return s;
  a.q = q; a.q_ld = q_ld; a.row_seq = row_seq; a.row_pos = row_pos; a.group = n_heads / a.c.hkv;
  a.budget = budget; a.keep_first = keep_first; a.keep_last = keep_last; a.ids = ids; a.status = status;
  cache_select_room(a.c, rows, workspace, &a);
  const bool bf = cache->dtype == DREAM_BF16;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const char *why = cache->head_dim == 64 ? (bf ? cache_select_run<bf16, 64>(a, rows, stream) : cache_select_run<f16, 64>(a, rows, stream))
                  : cache->head_dim == 128 ? (bf ? cache_select_run<bf16, 128>(a, rows, stream) : cache_select_run<f16, 128>(a, rows, stream))
                                           : (bf ? cache_select_run<bf16, 256>(a, rows, stream) : cache_select_run<f16, 256>(a, rows, stream));
  return why ? fail(nullptr, DREAM_E_CUDA, "%s: %s", who, why) : DREAM_OK;
}

// Most CTAs of the two attention kernels together, each of which may continue an item.
static int cache_slots(int hd) { return CACHE_MAX_SMS * (hd == 64 ? 3 : 2); }
// The parts of the attention's workspace; how many bytes they are.
static size_t cache_attn_room(const dream_cache *c, int n_heads, int rows, void *workspace, CacheAttnArgs *a) {
  const size_t n = 2 * (size_t)rows * n_heads, hd = c->head_dim;
  size_t at = 0;
  auto take = [&](size_t bytes) { char *p = (char *)workspace + at; at += (bytes + 255) / 256 * 256; return p; };
  char *po = take(n * hd * 4), *pm = take(n * 16), *co = take((size_t)cache_slots(c->head_dim) * 128 * hd * 4), *cm = take((size_t)cache_slots(c->head_dim) * 128 * 16);
  if (a) { a->part_o = (float *)po; a->part_ml = (float4 *)pm; a->cont_o = (float *)co; a->cont_ml = (float4 *)cm; }
  return at;
}

extern "C" dream_status dream_cache_attn_bytes(const dream_cache *cache, int32_t n_heads, int32_t rows, size_t *bytes) {
  CacheView v;
  dream_status s = cache_view("dream_cache_attn_bytes", cache, &v);
  if (!s) s = cache_heads("dream_cache_attn_bytes", cache, rows, n_heads);
  if (s) return s;
  if (!bytes) return fail(nullptr, DREAM_E_ARG, "dream_cache_attn_bytes: null argument");
  *bytes = cache_attn_room(cache, n_heads, rows, nullptr, nullptr);
  return DREAM_OK;
}

// What both attention calls ask for.
static dream_status cache_attn_args(const char *who, const dream_cache *cache, CacheAttnArgs *a, const void *q, long long q_ld, int n_heads, int rows, float scale,
                                    void *out, long long out_ld, float *lse, const void *workspace, size_t workspace_bytes, int *status) {
  size_t need = 0;
  dream_status s = cache_view(who, cache, &a->c);
  if (!s) s = cache_heads(who, cache, rows, n_heads);
  if (!s) s = cache_rows(who, "q", q, q_ld, (long long)n_heads * cache->head_dim);
  if (!s) s = cache_rows(who, "out", out, out_ld, (long long)n_heads * cache->head_dim);
  if (!s) s = cache_ints(who, "lse", lse, false);
  if (!s) s = cache_ints(who, "status", status, false);
  if (s) return s;
  if (!(scale > 0.f) || isinf(scale)) return fail(nullptr, DREAM_E_ARG, "%s: scale must be finite and above zero", who);
  if (rows_collide(q, q_ld, out, out_ld, DREAM_BF16, rows, n_heads * cache->head_dim) || q == out)
    return fail(nullptr, DREAM_E_ARG, "%s: out overlaps q", who);
  s = dream_cache_attn_bytes(cache, n_heads, rows, &need);
  if (!s) s = cache_workspace(who, workspace, workspace_bytes, need);
  if (s) return s;
  a->q = q; a->q_ld = q_ld; a->out = out; a->out_ld = out_ld; a->lse = lse; a->rows = rows; a->heads = n_heads; a->group = n_heads / a->c.hkv;
  a->scale_log2 = scale * 1.4426950408889634f; a->status = status;
  cache_attn_room(cache, n_heads, rows, const_cast<void *>(workspace), a);
  return DREAM_OK;
}
// A tensor of five dimensions as the copies take it, 64 columns (128 bytes, swizzled) at a time.
static const char *cache_map(int dtype, const void *base, const cuuint64_t (&dims)[5], const cuuint64_t (&strides)[4], const cuuint32_t (&box)[5], CUtensorMap *out) {
  static std::atomic<void *> found(nullptr);               // (by whichever thread comes first)
  void *fn = found.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult qr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qr) != cudaSuccess || !fn) { cudaGetLastError(); return "cuTensorMapEncodeTiled not available"; }
    found.store(fn, std::memory_order_release);
  }
  const PFN_cuTensorMapEncodeTiled_v12000 encode = (PFN_cuTensorMapEncodeTiled_v12000)fn;
  const cuuint32_t step[5] = {1, 1, 1, 1, 1};
  const CUresult r = encode(out, dtype == DREAM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, const_cast<void *>(base), dims, strides, box,
                            step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? nullptr : "the strides make no tensor map";
}
// K or V: the keys of one page that go into a unit of `unit`, and all panels of columns where they are the whole unit.
static const char *cache_kv_map(const dream_cache *c, const CacheView &v, const void *base, int unit, CUtensorMap *out) {
  const cuuint32_t sub = c->page_tokens < unit ? c->page_tokens : unit, panels = c->head_dim / 64;
  return cache_map(c->dtype, base, {64, (cuuint64_t)c->page_tokens, panels, (cuuint64_t)c->n_kv_heads, (cuuint64_t)c->n_pages},
                   {(cuuint64_t)v.token_stride * 2, 128, (cuuint64_t)v.head_stride * 2, (cuuint64_t)v.page_stride * 2},
                   {64, sub, sub == (cuuint32_t)unit ? panels : 1, 1, 1}, out);
}
// Q: a panel of so many rows' heads of one group, row after row, as a tile has its entries.
static const char *cache_q_map(const dream_cache *c, const CacheAttnArgs &a, int rows, CUtensorMap *out) {
  const cuuint64_t hd = c->head_dim;
  return cache_map(c->dtype, a.q, {64, hd / 64, (cuuint64_t)a.group, (cuuint64_t)c->n_kv_heads, (cuuint64_t)a.rows},
                   {128, hd * 2, a.group * hd * 2, (cuuint64_t)a.q_ld * 2}, {64, 1, (cuuint32_t)a.group, 1, (cuuint32_t)rows}, out);
}
// A kernel may use its shared memory on the current device from now on: once per device by a thread that calls again and again.  Returns the device's SMs, 0 with *e set
// where something is wrong.
template <typename... A>
static int cache_allow(void (*kernel)(A...), size_t smem, cudaError_t *e) {
  struct Ready { const void *kernel; int device, sms; };
  static thread_local Ready ready[16];
  static thread_local int next = 0;
  int device = 0, sms = 0;
  if ((*e = cudaGetDevice(&device)) != cudaSuccess) return 0;
  for (const Ready &r : ready) if (r.kernel == (const void *)kernel && r.device == device) return r.sms;
  *e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (*e == cudaSuccess) *e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (*e == cudaSuccess) *e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (*e != cudaSuccess) return 0;
  if (sms > CACHE_MAX_SMS) sms = CACHE_MAX_SMS;
  ready[next] = {(const void *)kernel, device, sms};
  next = (next + 1) % 16;
  return sms;
}
// Tiles of up to 128 entries.
template <typename T, int HD, bool PAGES>
static const char *cache_attn_many(const dream_cache *cache, CacheAttnArgs &a, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  const int sms = cache_allow(k_cache_attn<T, HD, PAGES>, CaShape<HD>::SMEM, &e);
  if (!sms) { cudaGetLastError(); return cudaGetErrorString(e); }
  CUtensorMap mk, mv, mq, ms;
  a.tile_rows = 128 / a.group;
  const char *why = cache_kv_map(cache, a.c, a.c.k, CaShape<HD>::BLK, &mk);
  if (!why) why = cache_kv_map(cache, a.c, a.c.v, CaShape<HD>::BLK, &mv);
  // a copy takes a whole tile of query entries, or 16 where a segment has no more
  a.q_small = a.group < 16 ? 16 / a.group : 1;
  if (!why) why = cache_q_map(cache, a, a.tile_rows, &mq);
  if (!why) why = cache_q_map(cache, a, a.q_small, &ms);
  if (why) return why;
  a.n_ctas = sms;
  a.cont_base = 0;
  return cache_launch(k_cache_attn<T, HD, PAGES>, dim3(a.n_ctas), CA_THREADS, CaShape<HD>::SMEM, stream, mk, mv, mq, ms, a);
}
// Tiles of up to CF_ENTRIES.
template <typename T, int HD, bool PAGES>
static const char *cache_attn_few(const dream_cache *cache, CacheAttnArgs &a, cudaStream_t stream) {
  using Sh = CfShape<HD>;
  cudaError_t e = cudaSuccess;
  const int sms = cache_allow(k_cache_attn_few<T, HD, PAGES>, Sh::SMEM, &e);
  if (!sms) { cudaGetLastError(); return cudaGetErrorString(e); }
  CUtensorMap mk, mv, mq;
  a.tile_rows = CF_ENTRIES / a.group;
  const char *why = cache_kv_map(cache, a.c, a.c.k, Sh::BLK, &mk);
  if (!why) why = cache_kv_map(cache, a.c, a.c.v, Sh::BLK, &mv);
  if (!why) why = cache_q_map(cache, a, a.tile_rows, &mq);
  if (why) return why;
  a.n_ctas = sms * Sh::CTAS_PER_SM;
  a.cont_base = CACHE_MAX_SMS;
  return cache_launch(k_cache_attn_few<T, HD, PAGES>, dim3(a.n_ctas), CF_THREADS, Sh::SMEM, stream, mk, mv, mq, a);
}
template <typename T, int HD, bool PAGES>
static const char *cache_attn_run(const dream_cache *cache, CacheAttnArgs &a, cudaStream_t stream) {
  // Query entries to a KV head: those of a listed row, or of all rows of a sequence.  How many rows a sequence has is on the device, so where sequences of up to four entries may stand
  // beside others (no more than four to a sequence on the average) both kernels are launched and each takes its own; but a call with as many rows as sequences and nothing shared is
  // taken to have a row of each.  (8 sequences of 20 rows in 256 slots, 32 heads over 8 of 128 behind 2000 tokens: 32 us, and 134 by the kernel for few alone; 63 tokens and a prompt
  // of 192 rows, 32 heads, 339 and 395.  What the other launch costs where it finds nothing: 64 slots with 8 rows 21.5 and 18, 16 sequences of 4 rows 55 and 52.)
  const long long entries = (long long)a.rows * a.group;
  const bool few = a.group <= CF_ENTRIES && (PAGES || entries <= (long long)CF_ENTRIES * a.c.n_seqs);
  const bool many = !few || (!PAGES && entries > CF_ENTRIES && (a.shared_tokens || a.rows != a.c.n_seqs));
  const char *why = nullptr;
  a.cont_slots = cache_slots(HD);
  auto launch_many = [&]() {
    if (why || !many) return;
    a.own_from = few ? CF_ENTRIES + 1 : 1; a.own_to = INT_MAX;
    a.with_prefix = a.shared_tokens > 0;
    why = cache_attn_many<T, HD, PAGES>(cache, a, stream);
  };
  auto launch_few = [&]() {
    if (why || !few) return;
    a.own_from = 1; a.own_to = many ? CF_ENTRIES : INT_MAX;
    a.with_prefix = !many && a.shared_tokens > 0;
    why = cache_attn_few<T, HD, PAGES>(cache, a, stream);
  };
  // In front, what there is most of: the shared keys, or those of single tokens.
  if (a.shared_tokens) {
    launch_many();
    a.early = few && many;
    launch_few();
  } else {
    a.let = few && many;
    launch_few();
    a.let = 0;
    a.early = few && many;
    launch_many();
  }
  // More (row, head)s than threads that merge them are resident at once: a CTA continues one item at most, so most of them are done already, unless each has two parts.  (Seven
  // sequences of 500 rows behind 4096 tokens 297 us, without the look 325; of 128 rows 90 and 88.)
  const long long rh = (long long)a.rows * a.heads, per = 256 / (HD / 4);
  a.look = (PAGES || !a.shared_tokens || entries >= 256LL * a.c.n_seqs) && rh > 148 * 8 * per;
  const long long blocks = a.look ? (rh + MERGE_LOOK - 1) / MERGE_LOOK : (rh + per - 1) / per;
  return why ? why : cache_launch(k_cache_merge<T, HD, PAGES>, dim3((unsigned)blocks), 256, 0, stream, a);
}
template <bool PAGES>
static const char *cache_attn_launch(const dream_cache *cache, CacheAttnArgs &a, cudaStream_t stream) {
  const bool b = cache->dtype == DREAM_BF16;
  if (cache->head_dim == 64) return b ? cache_attn_run<bf16, 64, PAGES>(cache, a, stream) : cache_attn_run<f16, 64, PAGES>(cache, a, stream);
  if (cache->head_dim == 128) return b ? cache_attn_run<bf16, 128, PAGES>(cache, a, stream) : cache_attn_run<f16, 128, PAGES>(cache, a, stream);
  return b ? cache_attn_run<bf16, 256, PAGES>(cache, a, stream) : cache_attn_run<f16, 256, PAGES>(cache, a, stream);
}

extern "C" dream_status dream_cache_attn(const dream_cache *cache, const void *q, int64_t q_ld, int32_t n_heads, int32_t rows, const int32_t *q_start,
                                         const int32_t *kv_len, int32_t shared_pages, const uint32_t *tree_mask, float scale, void *out, int64_t out_ld,
                                         float *lse, void *workspace, size_t workspace_bytes, int32_t *status, void *cuda_stream) {
  static const char who[] = "dream_cache_attn";
  CacheAttnArgs a = {};
  dream_status s = cache_attn_args(who, cache, &a, q, q_ld, n_heads, rows, scale, out, out_ld, lse, workspace, workspace_bytes, status);
  if (!s) s = cache_ints(who, "q_start", q_start, true);
  if (!s) s = cache_ints(who, "kv_len", kv_len, true);
  if (!s) s = cache_ints(who, "tree_mask", tree_mask, false);
  if (s) return s;
  if (shared_pages < 0 || shared_pages > cache->pages_per_seq) return fail(nullptr, DREAM_E_ARG, "%s: shared_pages = %d outside 0..pages_per_seq = %d", who, shared_pages, cache->pages_per_seq);
  a.q_start = q_start; a.kv_len = kv_len; a.tree = tree_mask;
  a.shared_tokens = shared_pages * cache->page_tokens;
  // The units of the prefix, those of one tile of a sequence and those of a CTA are counted in 32 bits (with what an item's start counts).
  auto units = [&](long long n_pages) { return (n_pages * cache->page_tokens / 64 + 1 + CF_START) * cache->n_kv_heads; };
  const int tile = 128 / a.group;                          // rows of one (CF_ENTRIES or fewer are one tile in either kernel)
  const long long tiles = (rows + tile - 1) / tile, few_tiles = a.group <= CF_ENTRIES && rows == cache->n_seqs ? rows : 0;      // (the kernel for few alone takes up to a row at a time)
  const long long own = units(cache->pages_per_seq), all = own * (tiles + cache->n_seqs + few_tiles) + (shared_pages ? units(shared_pages) * tiles : 0);
  if (own > 0x7fffffffLL || (shared_pages && units(shared_pages) * tiles > 0x7fffffffLL) || all / 128 > 0x7fffffffLL)      // (no fewer CTAs than that)
    return fail(nullptr, DREAM_E_CAPACITY, "%s: %d rows over sequences of %d pages in one call", who, rows, cache->pages_per_seq);
  const char *why = cache_attn_launch<false>(cache, a, (cudaStream_t)cuda_stream);
  return why ? fail(nullptr, DREAM_E_CUDA, "%s: %s", who, why) : DREAM_OK;
}

extern "C" dream_status dream_cache_attn_pages(const dream_cache *cache, const void *q, int64_t q_ld, int32_t n_heads, int32_t rows,
                                               const int32_t *row_seq, const int32_t *row_pos, const int32_t *ids, int32_t budget, float scale,
                                               void *out, int64_t out_ld, float *lse, void *workspace, size_t workspace_bytes, int32_t *status,
                                               void *cuda_stream) {
  static const char who[] = "dream_cache_attn_pages";
  CacheAttnArgs a = {};
  dream_status s = cache_attn_args(who, cache, &a, q, q_ld, n_heads, rows, scale, out, out_ld, lse, workspace, workspace_bytes, status);
  if (!s) s = cache_ints(who, "row_seq", row_seq, true);
  if (!s) s = cache_ints(who, "row_pos", row_pos, true);
  if (!s) s = cache_ints(who, "ids", ids, true);
  if (s) return s;
  if (budget < 1) return fail(nullptr, DREAM_E_ARG, "%s: budget = %d must be positive", who, budget);
  if (budget > CACHE_MAX_BUDGET) return fail(nullptr, DREAM_E_CAPACITY, "%s: budget above %d", who, CACHE_MAX_BUDGET);
  if ((long long)rows * cache->n_kv_heads > 0x7fffffffLL) return fail(nullptr, DREAM_E_CAPACITY, "%s: %d rows in one call", who, rows);
  a.row_seq = row_seq; a.row_pos = row_pos; a.ids = ids; a.budget = budget;
  const char *why = cache_attn_launch<true>(cache, a, (cudaStream_t)cuda_stream);
  return why ? fail(nullptr, DREAM_E_CUDA, "%s: %s", who, why) : DREAM_OK;
}
