// C ABI of libhswa: argument validation, layer-kind dispatch and host helpers.
// Every device call validates synchronously, then enqueues its kernels on the
// caller's stream; nothing here allocates device memory.
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "../../include/hswa.h"
#include "hswa_launch.h"

namespace {

bool sync_check_enabled() {
  static const bool on = [] {
    const char *e = std::getenv("HSWA_SYNC_CHECK");
    return e && e[0] && std::strcmp(e, "0") != 0;
  }();
  return on;
}

hswa_status finish_launch(hipError_t e, hipStream_t stream) {
  if (e != hipSuccess) return HSWA_ERR_LAUNCH;
  if (sync_check_enabled() && hipStreamSynchronize(stream) != hipSuccess) return HSWA_ERR_LAUNCH;
  return HSWA_OK;
}

int log2_exact(int32_t x) {
  if (x <= 0 || (x & (x - 1)) != 0) return -1;
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

constexpr int32_t kMaxKvHeads = 4096;
// (sequence, KV head) pairs of a call with a workgroup of up to 1024 threads for each: a grid
// holds less than 2^32 threads
constexpr int32_t kMaxGridRows = (1 << 22) - 1;
// (sequence, query, head) rows of the shared and scored decode, a merging wave for each, with
// up to 2^28 threads more beside them
constexpr int64_t kMaxRows = 1 << 25;
// Positions of a sequence whose sums of keys, tiles and spans stay within 32 bits
constexpr int32_t kMaxLen = 1 << 30;

// (their sizes of workspaces stay within 64 bits up to there)
bool too_many_rows(const hswa_shape *sh, int32_t ns, int32_t num_queries) {
  return (int64_t)ns * num_queries > kMaxRows / sh->num_q_heads;
}

// Shape checks shared by every device call.
hswa_status check_shape(const hswa_shape *sh) {
  if (!sh) return HSWA_ERR_INVALID_ARG;
  if (sh->num_q_heads <= 0 || sh->num_kv_heads <= 0 || sh->page_size <= 0 || sh->head_dim <= 0)
    return HSWA_ERR_INVALID_ARG;
  if (sh->num_q_heads % sh->num_kv_heads != 0) return HSWA_ERR_INVALID_ARG;
  if (!(sh->scale > 0.f) || !std::isfinite(sh->scale)) return HSWA_ERR_INVALID_ARG;
  if (sh->head_dim != hswa::kHeadDim) return HSWA_ERR_UNSUPPORTED;
  // a page-head of every KV head (Hkv * PG * D * 2 bytes) stays under 2^32,
  // which the kernels' 32-bit page strides assume
  if (sh->num_kv_heads > kMaxKvHeads) return HSWA_ERR_UNSUPPORTED;
  const int group = sh->num_q_heads / sh->num_kv_heads;
  if (128 % group != 0) return HSWA_ERR_UNSUPPORTED;
  const int s = log2_exact(sh->page_size);
  if (s < 4 || s > 8) return HSWA_ERR_UNSUPPORTED;
  return HSWA_OK;
}

hswa_status check_layer(hswa_layer layer) {
  if (layer.kind == HSWA_LAYER_FULL) return HSWA_OK;
  if (layer.kind == HSWA_LAYER_SWA || layer.kind == HSWA_LAYER_SWA_PAGED)
    return layer.window >= 1 ? HSWA_OK : HSWA_ERR_INVALID_ARG;
  return HSWA_ERR_INVALID_ARG;
}

// Builds the kernels' pool view; checks the pieces every call needs.
hswa_status make_pool(hswa_layer layer, const hswa_shape *sh, const hswa_cache *cache, hswa::PoolView &pv) {
  if (!cache || !cache->k_pool || !cache->v_pool || !cache->block_table) return HSWA_ERR_INVALID_ARG;
  if (cache->num_pages <= 0 || cache->table_stride <= 0) return HSWA_ERR_INVALID_ARG;
  pv.k_pool = static_cast<uint16_t *>(cache->k_pool);
  pv.v_pool = static_cast<uint16_t *>(cache->v_pool);
  pv.num_pages = cache->num_pages;
  pv.table = cache->block_table;
  pv.stride = cache->table_stride;
  pv.pg_shift = log2_exact(sh->page_size);
  pv.vb_shift = pv.pg_shift < hswa::kVBlockShiftMax ? pv.pg_shift : hswa::kVBlockShiftMax;
  if (layer.kind == HSWA_LAYER_SWA) {
    pv.ring = hswa_ring_pages(layer.window, sh->page_size);
    pv.window = layer.window;
    if (pv.ring > cache->table_stride) return HSWA_ERR_CAPACITY;
  } else if (layer.kind == HSWA_LAYER_SWA_PAGED) {  // FULL-style table, window masking
    pv.ring = 0;
    pv.window = layer.window;
  } else {
    pv.ring = 0;
    pv.window = 0;
  }
  return HSWA_OK;
}

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct DecodeGeometry {
  int32_t split_len;
  int32_t max_splits;
  size_t o_bytes;
  size_t total_bytes;
};

constexpr int32_t kMaxQueries = 64;  // queries per sequence in one decode call

// The first of nq new queries of an SWA layer reads the W - 1 keys before it,
// which must still be held once all nq tokens are appended. A ring keeps the
// latest R * PG positions, so nq <= R * PG - W + 1. An explicit-release table
// stores only the last W of the positions one extend adds, so nq <= W.
hswa_status check_multi_window(hswa_layer layer, const hswa_shape *sh, int32_t nq) {
  if (layer.kind == HSWA_LAYER_SWA) {
    const int64_t held = (int64_t)hswa_ring_pages(layer.window, sh->page_size) * sh->page_size;
    if ((int64_t)nq > held - layer.window + 1) return HSWA_ERR_UNSUPPORTED;
  } else if (layer.kind == HSWA_LAYER_SWA_PAGED) {
    if (nq > layer.window) return HSWA_ERR_UNSUPPORTED;
  }
  return HSWA_OK;
}

// `always`: split whatever the length (for calls that keep every row's
// log-sum-exp), by `shorter` keys where the rule's shortest spans, 256, are more.
DecodeGeometry decode_geometry(const hswa_shape *sh, int32_t ns, int32_t max_ctx, int32_t nq, bool always = false,
                               int32_t shorter = 256) {
  DecodeGeometry g{};
  const int group = sh->num_q_heads / sh->num_kv_heads;
  g.split_len = hswa::decode_split_len(ns, sh->num_kv_heads, group, max_ctx);
  if (max_ctx <= g.split_len && !always) {  // single pass, no workspace
    g.max_splits = 1;
    return g;
  }
  if (g.split_len == 256 && shorter < 256) g.split_len = shorter;
  // a segment of at most max_ctx keys meets at most ceil(max_ctx / split_len) + 1
  // spans of at least split_len keys
  g.max_splits = (max_ctx + g.split_len - 1) / g.split_len + 1;
  const size_t rows = (size_t)ns * nq * sh->num_q_heads * g.max_splits;
  g.o_bytes = align_up(rows * sh->head_dim * sizeof(float), 256);
  g.total_bytes = g.o_bytes + align_up(rows * sizeof(float), 256);
  return g;
}

// Shared-prefix decode: the plan, the partials of the own keys, those of the
// prefixes.
struct SharedGeometry {
  DecodeGeometry d;
  size_t groups, group_units, group_rows, own_units, start, group_of, seqs, own, ws_o, ws_lse, total_bytes;
};

SharedGeometry shared_geometry(const hswa_shape *sh, int32_t ns, int32_t max_ctx, int32_t nq, int32_t ng) {
  SharedGeometry g{};
  g.d = decode_geometry(sh, ns, max_ctx, nq, true, 128);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align_up(bytes, 256);
    return o;
  };
  take(sizeof(hswa::SharedHead));
  g.groups = take((size_t)ng * sizeof(hswa::SharedGroup));
  g.group_units = take(((size_t)ng + 1) * sizeof(int64_t));
  g.group_rows = take((size_t)ng * sizeof(int64_t));
  g.own_units = take((size_t)ns * sizeof(int64_t));
  g.start = take((size_t)ns * sizeof(int32_t));
  g.group_of = take((size_t)ns * sizeof(int32_t));
  g.seqs = take((size_t)ns * sizeof(hswa::SharedSeq));
  g.own = take(g.d.total_bytes);
  // a piece of a prefix has the rows of its columns, in 16s for a group's; each span adds at most a
  // workgroup's columns
  const size_t cols = (size_t)ns * nq * (sh->num_q_heads / sh->num_kv_heads);
  const size_t rows = sh->num_kv_heads * (cols + 15 * (size_t)ng) + (size_t)hswa::kSharedSpans * hswa::kSharedCols;
  g.ws_o = take(rows * sh->head_dim * sizeof(float));
  g.ws_lse = take(rows * sizeof(float));
  g.total_bytes = at;
  return g;
}

// Scored decode. Few columns: the split partials, then all scores. More: what
// shared-prefix decode takes with each sequence a group, then the rows'
// log-sum-exps.
struct ScoredGeometry {
  SharedGeometry s;
  bool keep;
  int64_t max_chunks;
  size_t front, total_bytes;
};

ScoredGeometry scored_geometry(const hswa_shape *sh, int32_t ns, int32_t max_ctx, int32_t nq) {
  ScoredGeometry g{};
  const size_t rows = (size_t)ns * nq * sh->num_q_heads;
  g.keep = nq * (sh->num_q_heads / sh->num_kv_heads) <= hswa::kKeepColumns;
  g.max_chunks = ((int64_t)max_ctx + 31) / 32;
  if (g.keep) {
    // Spans from 64 keys on where the batch does not fill the device's 1024 waves
    // with longer ones (the rows are merged in any case): 1 x 4K, 64 / 8 heads,
    // 13.5 us of decoding with 256, 10.5 with 64; 6 x 50 - 980, 8 / 1, 15.1 and 8.7.
    int32_t least = 64;
    while (least < 256 && (int64_t)sh->num_kv_heads * ns * max_ctx / least > 1024) least *= 2;
    g.s.d = decode_geometry(sh, ns, max_ctx, nq, true, least);
    g.front = g.s.d.total_bytes;
  } else {
    g.s = shared_geometry(sh, ns, max_ctx, nq, ns);
    g.front = g.s.total_bytes;
  }
  g.total_bytes = g.front + align_up(rows * sizeof(float) * (g.keep ? (size_t)g.max_chunks * 32 : 1), 256);
  return g;
}

// Whether a call goes by its prefixes: its plan, two ways of work and merge take
// some 12 us more than a short decode, which reading less has to make up for, at
// most (ns - num_groups) * max_shared_len positions of every KV head. us by prefix
// and by hswa_decode_multi, 100 - 300 own tokens, with the MB saved (shared keys):
//   64 / 8 heads   2 sequences x 8000      33 MB   23 / 22
//                  2 x 16000               66      25 / 34
//                  4 x 4000, 4 x 8000      49, 98  22 / 22, 24 / 31
//                  8 x 2000, 8 x 4000      57, 115 23 / 22, 23 / 31
//                  8 in 4 groups x 4000    66      28 / 33
//                  32 x 1000               127     27 / 33
//   8 / 1          8 x 16000, 8 x 32000    57, 115 21 / 21, 23 / 31
//                  32 x 4000               63      24 / 20
//   16 / 16        2 x 4000, 2 x 8000      33, 66  21 / 22, 24 / 31
//                  32 x 256                65      25 / 28
// (63 - 66 MB go both ways, so the limit stands above them: up to 9 us are given up
// there, rather than 4 lost.)
// Contexts of up to 256 keys, the shortest span, hswa_decode_multi takes in one pass
// and one launch, the shared pages out of the caches: of 113 such batches (8 - 400
// sequences, 64 - 250 shared keys, 1 - 8 queries) that save 70 MB and more, each took
// 1.06 to 6.4 times as long by prefix (64 / 8 heads, 84 sequences, 2 queries 51 / 9;
// 32 / 32, 336, 8 queries 443 / 89). Longer contexts over fewer than 256 shared keys
// go both ways (0.6 - 1.8), over 384 and more mostly one (0.27 - 1.43, 0.74 in the mean).
bool shared_fits(const hswa_shape *sh, int32_t ns, int32_t num_groups, int32_t max_context_len,
                 int32_t max_shared_len) {
  constexpr double kLeastSaved = 70e6;
  constexpr int32_t kOnePass = 256;
  if (ns < 2 || num_groups < 1 || max_shared_len < hswa::kSharedTile) return false;
  if (max_context_len <= kOnePass || max_context_len > kMaxLen) return false;
  const double keys = (double)(ns - num_groups) * (max_shared_len < max_context_len ? max_shared_len : max_context_len);
  return keys * sh->num_kv_heads * (sh->head_dim * 4) >= kLeastSaved;
}

// What every decode call tells its kernels besides the pool and the split.
void decode_params(hswa::DecodeParams &p, const hswa_shape *shape, const void *q, const int32_t *context_lens,
                   int32_t ns, int32_t num_queries, int32_t max_context_len, void *out) {
  p.q = static_cast<const uint16_t *>(q);
  p.ctx_lens = context_lens;
  p.out = static_cast<uint16_t *>(out);
  p.ns = ns;
  p.hq = shape->num_q_heads;
  p.hkv = shape->num_kv_heads;
  p.group = p.hq / p.hkv;
  p.max_ctx = max_context_len;
  p.nq = num_queries;
  p.scale_log2 = shape->scale * 1.4426950408889634f;
}

void split_params(hswa::DecodeParams &p, const DecodeGeometry &geo, char *ws) {
  p.split_len = geo.split_len;
  p.max_splits = geo.max_splits;
  p.ws_o = reinterpret_cast<float *>(ws);
  p.ws_lse = reinterpret_cast<float *>(ws + geo.o_bytes);
}

void shared_params(hswa::SharedParams &p, const SharedGeometry &geo, int32_t num_groups, char *ws) {
  split_params(p.d, geo.d, ws + geo.own);
  p.ng = num_groups;
  p.head = reinterpret_cast<hswa::SharedHead *>(ws);
  p.groups = reinterpret_cast<hswa::SharedGroup *>(ws + geo.groups);
  p.group_units = reinterpret_cast<int64_t *>(ws + geo.group_units);
  p.group_rows = reinterpret_cast<int64_t *>(ws + geo.group_rows);
  p.own_units = reinterpret_cast<int64_t *>(ws + geo.own_units);
  p.start = reinterpret_cast<int32_t *>(ws + geo.start);
  p.group_of = reinterpret_cast<int32_t *>(ws + geo.group_of);
  p.seqs = reinterpret_cast<hswa::SharedSeq *>(ws + geo.seqs);
  p.ws_o = reinterpret_cast<float *>(ws + geo.ws_o);
  p.ws_lse = reinterpret_cast<float *>(ws + geo.ws_lse);
  p.d.start = p.start;
  p.d.own_units = p.own_units;
  p.d.own = &p.head->own;
}

}  // namespace

extern "C" {

int32_t hswa_ring_pages(int32_t window, int32_t page_size) {
  if (window < 1 || page_size < 1) return -1;
  return (int32_t)(((int64_t)window + page_size - 1) / page_size + 1);
}

int64_t hswa_page_bytes(const hswa_shape *shape) {
  if (!shape || shape->num_kv_heads <= 0 || shape->page_size <= 0 || shape->head_dim <= 0) return -1;
  return (int64_t)shape->num_kv_heads * shape->page_size * shape->head_dim * 2;
}

hswa_status hswa_build_block_table(hswa_layer layer, int32_t page_size, int32_t ns, const int32_t *final_lens,
                                   const int32_t *perm, int64_t perm_len, int32_t *table_out, int32_t stride) {
  if (check_layer(layer) != HSWA_OK || page_size < 1 || ns < 0 || stride < 1 || perm_len < 0)
    return HSWA_ERR_INVALID_ARG;
  if (ns > 0 && (!final_lens || !table_out)) return HSWA_ERR_INVALID_ARG;
  if (perm_len > 0 && !perm) return HSWA_ERR_INVALID_ARG;
  int64_t off = 0;
  for (int32_t b = 0; b < ns; ++b) {
    if (final_lens[b] < 0) return HSWA_ERR_INVALID_ARG;
    const int64_t need = layer.kind == HSWA_LAYER_SWA ? hswa_ring_pages(layer.window, page_size)
                                                      : ((int64_t)final_lens[b] + page_size - 1) / page_size;
    if (need > stride || off + need > perm_len) return HSWA_ERR_CAPACITY;
    int32_t *row = table_out + (int64_t)b * stride;
    for (int64_t i = 0; i < stride; ++i) row[i] = i < need ? perm[off + i] : -1;
    off += need;
  }
  return HSWA_OK;
}

hswa_status hswa_kv_append(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *k_new,
                           const void *v_new, const int32_t *cu_seqlens, const int32_t *start_pos, int32_t ns,
                           int32_t total_tokens, int64_t *slot_mapping_out, void *stream) {
  hswa_status st;
  if ((st = check_layer(layer)) != HSWA_OK) return st;
  if ((st = check_shape(shape)) != HSWA_OK) return st;
  if (ns < 0 || total_tokens < 0) return HSWA_ERR_INVALID_ARG;
  hswa::PoolView pv{};
  if ((st = make_pool(layer, shape, cache, pv)) != HSWA_OK) return st;
  if (ns == 0 || total_tokens == 0) return HSWA_OK;
  if (!k_new || !v_new || !cu_seqlens || !start_pos) return HSWA_ERR_INVALID_ARG;
  hswa::AppendParams p{};
  p.pool = pv;
  p.k_new = static_cast<const uint16_t *>(k_new);
  p.v_new = static_cast<const uint16_t *>(v_new);
  p.cu_seqlens = cu_seqlens;
  p.start_pos = start_pos;
  p.slot_out = slot_mapping_out;
  p.ns = ns;
  p.total_tokens = total_tokens;
  p.hkv = shape->num_kv_heads;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return finish_launch(hswa::launch_kv_append(p, s), s);
}

hswa_status hswa_prefill(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                         const void *k_new, const void *v_new, const int32_t *cu_seqlens, const int32_t *prefix_lens,
                         int32_t ns, int32_t total_tokens, int32_t max_chunk_len, void *out, void *stream) {
  return hswa_prefill_ws(layer, shape, cache, q, k_new, v_new, cu_seqlens, prefix_lens, ns, total_tokens,
                         max_chunk_len, nullptr, 0, out, stream);
}

size_t hswa_prefill_workspace_bytes(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, int32_t ns,
                                    int32_t total_tokens, int32_t max_chunk_len) {
  hswa::PrefillParams p{};
  if (check_layer(layer) != HSWA_OK || check_shape(shape) != HSWA_OK) return 0;
  if (make_pool(layer, shape, cache, p.pool) != HSWA_OK) return 0;
  p.ns = ns;
  p.total_tokens = total_tokens;
  p.max_chunk_len = max_chunk_len;
  p.hkv = shape->num_kv_heads;
  p.group = shape->num_q_heads / p.hkv;
  return hswa::prefill_split_fits(p) ? hswa::prefill_split_bytes() : 0;
}

hswa_status hswa_prefill_ws(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                            const void *k_new, const void *v_new, const int32_t *cu_seqlens,
                            const int32_t *prefix_lens, int32_t ns, int32_t total_tokens, int32_t max_chunk_len,
                            void *workspace, size_t workspace_bytes, void *out, void *stream) {
  hswa_status st;
  if ((st = check_layer(layer)) != HSWA_OK) return st;
  if ((st = check_shape(shape)) != HSWA_OK) return st;
  if (ns < 0 || total_tokens < 0 || max_chunk_len < 0) return HSWA_ERR_INVALID_ARG;
  hswa::PoolView pv{};
  if ((st = make_pool(layer, shape, cache, pv)) != HSWA_OK) return st;
  if (ns == 0 || total_tokens == 0 || max_chunk_len == 0) return HSWA_OK;
  if (!q || !k_new || !v_new || !cu_seqlens || !prefix_lens || !out) return HSWA_ERR_INVALID_ARG;
  hswa::PrefillParams p{};
  p.pool = pv;
  p.q = static_cast<const uint16_t *>(q);
  p.k_new = static_cast<const uint16_t *>(k_new);
  p.v_new = static_cast<const uint16_t *>(v_new);
  p.cu_seqlens = cu_seqlens;
  p.prefix_lens = prefix_lens;
  p.out = static_cast<uint16_t *>(out);
  p.ns = ns;
  p.total_tokens = total_tokens;
  p.max_chunk_len = max_chunk_len;
  p.hq = shape->num_q_heads;
  p.hkv = shape->num_kv_heads;
  p.group = p.hq / p.hkv;
  p.scale_log2 = shape->scale * 1.4426950408889634f;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (workspace && hswa::prefill_split_fits(p)) {
    if (workspace_bytes < hswa::prefill_split_bytes()) return HSWA_ERR_CAPACITY;
    return finish_launch(hswa::launch_prefill_split(p, workspace, s), s);
  }
  return finish_launch(hswa::launch_prefill(p, s), s);
}

size_t hswa_decode_multi_workspace_bytes(const hswa_shape *shape, int32_t ns, int32_t num_queries,
                                         int32_t max_context_len) {
  if (check_shape(shape) != HSWA_OK || ns < 0 || max_context_len < 1) return 0;
  if (num_queries < 1 || num_queries > kMaxQueries) return 0;
  if (ns == 0) return 0;
  return decode_geometry(shape, ns, max_context_len, num_queries).total_bytes;
}

size_t hswa_decode_workspace_bytes(const hswa_shape *shape, int32_t ns, int32_t max_context_len) {
  return hswa_decode_multi_workspace_bytes(shape, ns, 1, max_context_len);
}

int32_t hswa_decode_split_len(const hswa_shape *shape, int32_t ns, int32_t max_context_len) {
  if (check_shape(shape) != HSWA_OK || ns < 1 || max_context_len < 1) return -1;
  return decode_geometry(shape, ns, max_context_len, 1).split_len;
}

}  // extern "C"

namespace {

// Shared body of the decode entry points. With `noalloc` the FULL split
// partials go to the library's fixed device array instead of `workspace`.
// With k_new / v_new (one query per sequence) the call first stores the step's
// new token of every sequence, in the same launch when the kernel allows it.
hswa_status decode_impl(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                        const int32_t *context_lens, int32_t ns, int32_t num_queries, int32_t max_context_len,
                        void *workspace, size_t workspace_bytes, bool noalloc, void *out, void *stream,
                        const void *k_new = nullptr, const void *v_new = nullptr, bool append = false) {
  hswa_status st;
  if ((st = check_layer(layer)) != HSWA_OK) return st;
  if ((st = check_shape(shape)) != HSWA_OK) return st;
  if (ns < 0 || max_context_len < 1 || num_queries < 1 || num_queries > kMaxQueries) return HSWA_ERR_INVALID_ARG;
  hswa::PoolView pv{};
  if ((st = make_pool(layer, shape, cache, pv)) != HSWA_OK) return st;
  if ((st = check_multi_window(layer, shape, num_queries)) != HSWA_OK) return st;
  // FULL-style tables are indexed by the logical page of every position
  if ((layer.kind == HSWA_LAYER_FULL || layer.kind == HSWA_LAYER_SWA_PAGED) &&
      (int64_t)cache->table_stride * shape->page_size < (int64_t)max_context_len)
    return HSWA_ERR_CAPACITY;
  if (ns == 0) return HSWA_OK;
  if (!q || !context_lens || !out) return HSWA_ERR_INVALID_ARG;
  if (append && (!k_new || !v_new)) return HSWA_ERR_INVALID_ARG;
  hswa::DecodeParams p{};
  p.pool = pv;
  decode_params(p, shape, q, context_lens, ns, num_queries, max_context_len, out);
  if (layer.kind == HSWA_LAYER_FULL) {
    const DecodeGeometry geo = decode_geometry(shape, ns, max_context_len, num_queries);
    p.split_len = geo.split_len;
    p.max_splits = geo.max_splits;
    if (geo.max_splits > 1) {
      if (noalloc) {
        if (geo.total_bytes > HSWA_NOALLOC_SCRATCH_BYTES) return HSWA_ERR_CAPACITY;
        if (hswa::noalloc_scratch(&workspace) != hipSuccess) return HSWA_ERR_LAUNCH;
      } else {
        if (!workspace) return HSWA_ERR_INVALID_ARG;
        if (workspace_bytes < geo.total_bytes) return HSWA_ERR_CAPACITY;
      }
      p.ws_o = static_cast<float *>(workspace);
      p.ws_lse = reinterpret_cast<float *>(static_cast<char *>(workspace) + geo.o_bytes);
    }
  } else {
    p.split_len = max_context_len;
    p.max_splits = 1;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (append) {
    p.k_new = static_cast<const uint16_t *>(k_new);
    p.v_new = static_cast<const uint16_t *>(v_new);
    if (hswa::decode_append_fused(p)) return finish_launch(hswa::launch_decode_append(p, s), s);
    if (p.max_splits > 1 && p.nq == 1) {
      // FULL split path: the split decode stores the token itself
      p.split_append = 1;
      return finish_launch(hswa::launch_decode(p, s), s);
    }
    hswa::AppendParams a{};
    a.pool = pv;
    a.k_new = p.k_new;
    a.v_new = p.v_new;
    a.ns = ns;
    a.total_tokens = ns;
    a.hkv = p.hkv;
    a.ctx_lens = context_lens;
    a.max_ctx = max_context_len;
    const hipError_t e = hswa::launch_kv_append(a, s);
    if (e != hipSuccess) return HSWA_ERR_LAUNCH;
  }
  return finish_launch(hswa::launch_decode(p, s), s);
}

}  // namespace

extern "C" {

hswa_status hswa_decode_multi(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                              const int32_t *context_lens, int32_t ns, int32_t num_queries, int32_t max_context_len,
                              void *workspace, size_t workspace_bytes, void *out, void *stream) {
  return decode_impl(layer, shape, cache, q, context_lens, ns, num_queries, max_context_len, workspace,
                     workspace_bytes, false, out, stream);
}

hswa_status hswa_decode(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                        const int32_t *context_lens, int32_t ns, int32_t max_context_len, void *workspace,
                        size_t workspace_bytes, void *out, void *stream) {
  return decode_impl(layer, shape, cache, q, context_lens, ns, 1, max_context_len, workspace, workspace_bytes, false,
                     out, stream);
}

hswa_status hswa_decode_append(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                               const void *k_new, const void *v_new, const int32_t *context_lens, int32_t ns,
                               int32_t max_context_len, void *workspace, size_t workspace_bytes, void *out,
                               void *stream) {
  return decode_impl(layer, shape, cache, q, context_lens, ns, 1, max_context_len, workspace, workspace_bytes, false,
                     out, stream, k_new, v_new, true);
}

hswa_status hswa_decode_noalloc(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                                const int32_t *context_lens, int32_t ns, int32_t max_context_len, void *out,
                                void *stream) {
  return decode_impl(layer, shape, cache, q, context_lens, ns, 1, max_context_len, nullptr, 0, true, out, stream);
}

size_t hswa_decode_shared_workspace_bytes(const hswa_shape *shape, int32_t ns, int32_t num_queries,
                                          int32_t max_context_len, int32_t num_groups, int32_t max_shared_len) {
  if (check_shape(shape) != HSWA_OK || ns < 1 || max_context_len < 1 || num_groups < 0 || num_groups > ns) return 0;
  if (num_queries < 1 || num_queries > kMaxQueries || max_shared_len < 0) return 0;
  if (!shared_fits(shape, ns, num_groups, max_context_len, max_shared_len))
    return hswa_decode_multi_workspace_bytes(shape, ns, num_queries, max_context_len);
  if (too_many_rows(shape, ns, num_queries)) return 0;
  return shared_geometry(shape, ns, max_context_len, num_queries, num_groups).total_bytes;
}

hswa_status hswa_decode_shared(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                               const int32_t *context_lens, int32_t ns, int32_t num_queries, int32_t max_context_len,
                               const int32_t *cu_groups, const int32_t *shared_lens, int32_t num_groups,
                               int32_t max_shared_len, void *workspace, size_t workspace_bytes, void *out,
                               void *stream) {
  if (num_groups < 0 || max_shared_len < 0 || (ns >= 0 && num_groups > ns)) return HSWA_ERR_INVALID_ARG;
  if (num_groups > 0 && (!cu_groups || !shared_lens)) return HSWA_ERR_INVALID_ARG;
  if (layer.kind != HSWA_LAYER_FULL || check_shape(shape) != HSWA_OK ||
      !shared_fits(shape, ns, num_groups, max_context_len, max_shared_len))
    return hswa_decode_multi(layer, shape, cache, q, context_lens, ns, num_queries, max_context_len, workspace,
                             workspace_bytes, out, stream);
  hswa_status st;
  if (max_context_len < 1 || num_queries < 1 || num_queries > kMaxQueries) return HSWA_ERR_INVALID_ARG;
  hswa::SharedParams p{};
  if ((st = make_pool(layer, shape, cache, p.d.pool)) != HSWA_OK) return st;
  if ((int64_t)cache->table_stride * shape->page_size < (int64_t)max_context_len) return HSWA_ERR_CAPACITY;
  if (!q || !context_lens || !out || !workspace) return HSWA_ERR_INVALID_ARG;
  if (too_many_rows(shape, ns, num_queries)) return HSWA_ERR_UNSUPPORTED;
  const SharedGeometry geo = shared_geometry(shape, ns, max_context_len, num_queries, num_groups);
  if (workspace_bytes < geo.total_bytes) return HSWA_ERR_CAPACITY;
  decode_params(p.d, shape, q, context_lens, ns, num_queries, max_context_len, out);
  shared_params(p, geo, num_groups, static_cast<char *>(workspace));
  p.cu_groups = cu_groups;
  p.shared_lens = shared_lens;
  p.max_shared = max_shared_len;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return finish_launch(hswa::launch_decode_shared(p, s), s);
}

size_t hswa_decode_scored_workspace_bytes(const hswa_shape *shape, int32_t ns, int32_t num_queries,
                                          int32_t max_context_len) {
  if (check_shape(shape) != HSWA_OK || ns < 1 || max_context_len < 1) return 0;
  if (num_queries < 1 || num_queries > kMaxQueries || max_context_len > kMaxLen) return 0;
  if (too_many_rows(shape, ns, num_queries)) return 0;
  return scored_geometry(shape, ns, max_context_len, num_queries).total_bytes;
}

hswa_status hswa_decode_scored(hswa_layer layer, const hswa_shape *shape, const hswa_cache *cache, const void *q,
                               const int32_t *context_lens, int32_t ns, int32_t num_queries, int32_t max_context_len,
                               const float *scores_in, float *scores_out, int32_t score_stride, void *workspace,
                               size_t workspace_bytes, void *out, void *stream) {
  hswa_status st;
  if ((st = check_layer(layer)) != HSWA_OK) return st;
  if ((st = check_shape(shape)) != HSWA_OK) return st;
  if (layer.kind != HSWA_LAYER_FULL) return HSWA_ERR_UNSUPPORTED;
  if (ns < 0 || max_context_len < 1 || num_queries < 1 || num_queries > kMaxQueries) return HSWA_ERR_INVALID_ARG;
  if (max_context_len > kMaxLen) return HSWA_ERR_UNSUPPORTED;
  hswa::ScoredParams p{};
  if ((st = make_pool(layer, shape, cache, p.s.d.pool)) != HSWA_OK) return st;
  if ((int64_t)cache->table_stride * shape->page_size < (int64_t)max_context_len) return HSWA_ERR_CAPACITY;
  if (score_stride < max_context_len) return HSWA_ERR_CAPACITY;
  if (ns == 0) return HSWA_OK;
  if (!q || !context_lens || !out || !scores_out || !workspace) return HSWA_ERR_INVALID_ARG;
  if (too_many_rows(shape, ns, num_queries)) return HSWA_ERR_UNSUPPORTED;
  const ScoredGeometry geo = scored_geometry(shape, ns, max_context_len, num_queries);
  if (workspace_bytes < geo.total_bytes) return HSWA_ERR_CAPACITY;
  decode_params(p.s.d, shape, q, context_lens, ns, num_queries, max_context_len, out);
  char *ws = static_cast<char *>(workspace);
  if (geo.keep) {
    split_params(p.s.d, geo.s.d, ws);
    p.s.d.ws_s = reinterpret_cast<float *>(ws + geo.front);
    p.s.d.max_chunks = geo.max_chunks;
  } else {
    shared_params(p.s, geo.s, ns, ws);
    p.s.max_shared = max_context_len;
    p.s.d.row_lse = reinterpret_cast<float *>(ws + geo.front);
  }
  p.scores_in = scores_in;
  p.scores_out = scores_out;
  p.stride = score_stride;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return finish_launch(hswa::launch_decode_scored(p, s), s);
}

hswa_status hswa_kv_evict(hswa_layer layer, const hswa_shape *shape, const hswa_cache *src, const hswa_cache *dst,
                          const float *scores, int32_t score_stride, const int32_t *context_lens,
                          const int32_t *budgets, int32_t ns, int32_t max_context_len, int32_t num_recent,
                          int32_t num_sinks, int32_t *kept_out, int32_t kept_stride, float *scores_out,
                          int32_t scores_out_stride, int32_t *new_lens_out, void *stream) {
  hswa_status st;
  if ((st = check_layer(layer)) != HSWA_OK) return st;
  if ((st = check_shape(shape)) != HSWA_OK) return st;
  if (layer.kind != HSWA_LAYER_FULL) return HSWA_ERR_UNSUPPORTED;
  if (ns < 0 || max_context_len < 1 || num_recent < 0 || num_sinks < 0 || kept_stride < 1) return HSWA_ERR_INVALID_ARG;
  if (ns > kMaxGridRows / shape->num_kv_heads) return HSWA_ERR_UNSUPPORTED;
  if (max_context_len > kMaxLen || kept_stride > kMaxLen) return HSWA_ERR_UNSUPPORTED;
  hswa::EvictParams p{};
  if ((st = make_pool(layer, shape, src, p.src)) != HSWA_OK) return st;
  if ((st = make_pool(layer, shape, dst, p.dst)) != HSWA_OK) return st;
  const int64_t pg = shape->page_size;
  if (src->table_stride * pg < max_context_len || dst->table_stride * pg < kept_stride) return HSWA_ERR_CAPACITY;
  if (score_stride < max_context_len || (scores_out && scores_out_stride < kept_stride)) return HSWA_ERR_CAPACITY;
  if (src->block_table == dst->block_table) return HSWA_ERR_INVALID_ARG;
  if (ns == 0) return HSWA_OK;
  if (!scores || !context_lens || !budgets || !kept_out || !new_lens_out || scores_out == scores)
    return HSWA_ERR_INVALID_ARG;
  // (each KV head's workgroup reads the lengths and budgets, one of them writes the new lengths)
  if (new_lens_out == context_lens || new_lens_out == budgets) return HSWA_ERR_INVALID_ARG;
  p.scores = scores;
  p.ctx_lens = context_lens;
  p.budgets = budgets;
  p.kept = kept_out;
  p.scores_out = scores_out;
  p.new_lens = new_lens_out;
  p.score_stride = score_stride;
  p.out_stride = scores_out_stride;
  p.ns = ns;
  p.hkv = shape->num_kv_heads;
  p.max_ctx = max_context_len;
  p.max_keep = kept_stride;
  p.num_recent = num_recent;
  p.num_sinks = num_sinks;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return finish_launch(hswa::launch_kv_evict(p, s), s);
}

const char *hswa_status_string(hswa_status status) {
  switch (status) {
    case HSWA_OK: return "HSWA_OK";
    case HSWA_ERR_INVALID_ARG: return "HSWA_ERR_INVALID_ARG";
    case HSWA_ERR_UNSUPPORTED: return "HSWA_ERR_UNSUPPORTED";
    case HSWA_ERR_CAPACITY: return "HSWA_ERR_CAPACITY";
    case HSWA_ERR_LAUNCH: return "HSWA_ERR_LAUNCH";
  }
  return "HSWA_UNKNOWN_STATUS";
}

}  // extern "C"
