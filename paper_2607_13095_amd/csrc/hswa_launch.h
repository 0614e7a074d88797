// Internal launcher interface between the C ABI layer (api.hip) and the
// kernels. Arguments are validated by the caller before these are reached.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hswa {

constexpr int kHeadDim = 128;  // the only head dim the kernels are built for
constexpr int kHeadDimShift = 7;
// Both pools store a page-head as PG / B blocks of B = min(PG, 32) consecutive
// keys. V blocks are transposed ([D][B]): the V^T operand of a 32-key chunk of
// one head is one contiguous 8 KiB run. K blocks hold two halves (keys whose
// in-block offset has bit 2 clear, then set), each as four 32-dim slabs of
// [B/2 keys][32 dims] with the 16-byte pieces in bf16-MFMA lane order: the 16
// keys x 32 dims of one QK^T operand are one contiguous 1 KiB run (B = 32).
constexpr int kVBlockShiftMax = 5;

// Pool geometry and block table of one layer, as the kernels see it.
struct PoolView {
  uint16_t *k_pool;       // bf16 [num_pages][Hkv][PG/B][2][D/32][4][B/2][8]
  uint16_t *v_pool;       // bf16 [num_pages][Hkv][PG/B][D][B]
  int64_t num_pages;
  const int32_t *table;   // int32 [ns][stride]
  int32_t stride;
  int32_t pg_shift;       // log2(page size)
  int32_t vb_shift;       // log2(B) = min(pg_shift, 5), the key block of both pools
  int32_t ring;           // ring pages R (SWA) or 0 (FULL)
  int32_t window;         // SWA window W, or 0 for FULL
};

struct AppendParams {
  PoolView pool;
  const uint16_t *k_new;  // [T][Hkv][D]
  const uint16_t *v_new;  // [T][Hkv][D]
  const int32_t *cu_seqlens;
  const int32_t *start_pos;
  int64_t *slot_out;      // [T] or null
  int32_t ns, total_tokens, hkv;
  // Decode-step mode (ctx_lens non-null): token b is sequence b's, at position
  // min(ctx_lens[b], max_ctx) - 1 (none if that is negative); cu_seqlens and
  // start_pos are not read.
  const int32_t *ctx_lens;
  int32_t max_ctx;
};

// Suffix decode: the order of spans. Every (sequence, KV head and column item)
// takes its chunks in units, or with `aligned` those rounded up to whole spans (a
// span then belongs to one of them).
struct OwnSpans {
  int64_t units;
  int64_t per;  // of a span
  int32_t aligned;
};

struct DecodeParams {
  PoolView pool;
  const uint16_t *q;      // [ns][Hq][D]
  const int32_t *ctx_lens;
  uint16_t *out;          // [ns][Hq][D]
  float *ws_o;            // FULL split partials [ns * nq * Hq][max_splits][D]
  float *ws_lse;          // [ns * nq * Hq][max_splits]
  int32_t ns, hq, hkv, group, max_ctx;
  int32_t nq;             // queries per sequence, at positions ctx - nq .. ctx - 1 (q, out: [ns][nq][Hq][D])
  int32_t split_len;      // FULL split: fewest keys of a wave's span (a multiple of 32)
  int32_t max_splits;     // pieces a (row) may have; 1 => single pass, no workspace
  int32_t span_waves;     // FULL split: waves the chunk order is divided over (set at launch)
  int32_t item_cols;      // (query, head) columns of one item (set at launch)
  float scale_log2;       // scale * log2(e)
  const uint16_t *k_new;  // decode step: the new token's K / V rows [ns][Hkv][D]
  const uint16_t *v_new;
  // FULL split decode of one new token per sequence: the kernel also
  // stores the token (k_new / v_new) in its slot and takes its key from them
  int32_t split_append;
  float *row_lse;             // scored decode: [ns * nq * Hq], the rows' log2 sum-exps
  // or all scores in exp2 units, [ns][Hkv][max_chunks][nq * group][32]
  float *ws_s;
  int64_t max_chunks;         // 32-key chunks of max_ctx
  const int32_t *start;       // suffix decode: [ns], first key (a multiple of 32) of each sequence
  const int64_t *own_units;   // [ns] units before each sequence's in the order of spans
  const OwnSpans *own;
};

// Split prefill: the query tile at the start of a span, for the merge.
struct PrefillDesc {
  int32_t pieces;     // spans that met the tile; 0: nothing to merge here
  int32_t tok;        // first token of the tile
  int32_t positions;  // its positions
  int32_t head;       // KV head
};

struct PrefillParams {
  PoolView pool;
  const uint16_t *q;      // [T][Hq][D]
  const uint16_t *k_new;  // [T][Hkv][D]
  const uint16_t *v_new;  // [T][Hkv][D]
  const int32_t *cu_seqlens;
  const int32_t *prefix_lens;
  uint16_t *out;          // [T][Hq][D]
  int32_t ns, total_tokens, max_chunk_len, hq, hkv, group;
  float scale_log2;
  float *ws_o;            // split: partial outputs [2 spans][256 rows][D], in accumulator order
  float *ws_lse;          // [2 spans][256 rows]
  PrefillDesc *ws_desc;   // [spans]
};

// Decode over shared prefixes (decode_shared.hip). The plan, in the workspace:
constexpr int kSharedTile = 64;    // keys of a tile of the prefix
constexpr int kSharedCols = 256;   // (sequence, query, head) columns of a workgroup
constexpr int kSharedSpans = 256;  // workgroups of the work kernel, one per compute unit
struct SharedGroup {
  int32_t first;   // its first sequence
  int32_t leader;  // the first with a context: the prefix is read from its row of the table
  int32_t tiles;   // key tiles taken as shared (0: none)
  int32_t padded;  // units that they take in the order of spans
  int32_t cols;    // columns of a KV head (0 without tiles)
};
// What the merge needs of a sequence.
struct SharedSeq {
  int32_t start;           // shared keys
  int32_t col;             // its first column in its group's
  int32_t tiles, padded, cols;  // of its group
  int64_t units, rows;     // before its group
  int64_t own_units;
};
struct SharedHead {
  int64_t units;    // key tiles of all (group, KV head, kSharedCols columns), padded
  int64_t per;      // of them, those of a span
  OwnSpans own;
  int32_t prefix_groups;  // workgroups on key tiles of prefixes (a multiple of 8); the rest take own keys
};
struct SharedParams {
  DecodeParams d;              // the own keys; start, own_units and own point into the plan
  const int32_t *cu_groups;    // [ng + 1], or null: every sequence is a group, all it can share
  const int32_t *shared_lens;  // [ng]
  int32_t ng, max_shared;
  int32_t small;               // the workgroups find the plan (set at launch)
  SharedHead *head;
  SharedGroup *groups;   // [ng]
  int64_t *group_units;  // [ng + 1] units before each group
  int64_t *group_rows;   // [ng] rows of partials before each group
  int64_t *own_units;    // [ns] units of own keys (of every KV head) before each sequence's
  int32_t *start;        // [ns] shared keys of each sequence
  int32_t *group_of;     // [ns] (batches whose plan is a kernel)
  SharedSeq *seqs;       // [ns]
  float *ws_o;           // partial rows of the prefixes
  float *ws_lse;
};

// Decode that also adds every key's attention weight to a score (decode_scored.hip).
// Up to this many (query, head) columns of a KV head, one column group of a wave,
// the scores are stored: 4 bytes for each column of a key, for max_ctx keys of every
// sequence whatever its length. 64 / 8 heads, 16 sequences, us a call with them
// stored (by two column groups a wave) and formed anew: 24 columns (3 queries) over
// 2 - 16K keys 186 and 213, over 30 - 32K 558 and 567; 32 columns 205 and 216, 620
// and 570. So 17 - 24 columns would gain 2 - 13% by storing, and 32 lose 9% on long
// contexts; both are formed anew for the workspace's sake, which takes 0.54 GB for
// 16 columns of 16 x 64K keys already, and would take 0.8 and 1.1.
constexpr int kKeepColumns = 16;
struct ScoredParams {
  SharedParams s;          // s.d: split, with ws_s; or with row_lse, all of s, each sequence a group
  const float *scores_in;  // [ns][Hkv][stride], or null for zeros; may be scores_out
  float *scores_out;
  int64_t stride;
  int64_t merge_blocks;    // workgroups that merge rows (set at launch)
};

// Eviction (kv_evict.hip): keys of `src` kept by score move to the pages of `dst`.
struct EvictParams {
  PoolView src, dst;
  const float *scores;      // [ns][Hkv][score_stride]
  const int32_t *ctx_lens;  // [ns]
  const int32_t *budgets;   // [ns] keys to keep
  int32_t *kept;            // [ns][Hkv][max_keep] kept positions, in order
  float *scores_out;        // [ns][Hkv][out_stride] scores of the kept keys, or null
  int32_t *new_lens;        // [ns]
  int64_t score_stride, out_stride;
  int32_t ns, hkv, max_ctx, max_keep, num_recent, num_sinks;
};

hipError_t launch_kv_append(const AppendParams &p, hipStream_t stream);
hipError_t launch_decode_shared(const SharedParams &p, hipStream_t stream);
// The same with fp32 row sums, leaving the rows' log2 sum-exps in d.row_lse.
hipError_t launch_decode_shared_scored(const SharedParams &p, hipStream_t stream);
hipError_t launch_decode_scored(const ScoredParams &p, hipStream_t stream);
hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream);
hipError_t launch_decode(const DecodeParams &p, hipStream_t stream);
// Decode step with its append in the same launch (decode_append.hip): one
// query per sequence, whole-range items of at most 8 chunks.
bool decode_append_fused(const DecodeParams &p);
hipError_t launch_decode_append(const DecodeParams &p, hipStream_t stream);
hipError_t launch_prefill(const PrefillParams &p, hipStream_t stream);
// FULL prefill that may be cut into equal spans of key tiles (prefill.hip):
// whether a call can gain from it, the workspace it takes (any call), the launch.
bool prefill_split_fits(const PrefillParams &p);
size_t prefill_split_bytes();
hipError_t launch_prefill_split(const PrefillParams &p, void *workspace, hipStream_t stream);
// SWA prefill whose window is at most kPrefillWindowMax keys: 128 query rows
// per workgroup over the window's keys only (prefill_window.hip).
constexpr int kPrefillWindowMax = 512;
hipError_t launch_prefill_window(const PrefillParams &p, hipStream_t stream);
// SWA prefill with a GQA group of at least 8 and W + 256 / G - 1 <= 160: one
// workgroup per run of position tiles, the window's chunks in an LDS ring
// (prefill_run.hip).
bool prefill_run_fits(const PrefillParams &p);
hipError_t launch_prefill_run(const PrefillParams &p, hipStream_t stream);

// Device address of the library's fixed scratch array on the current device
// (looked up once per device).
hipError_t noalloc_scratch(void **ptr);

// Fewest keys of a FULL decode wave's span; a multiple of 256.
int32_t decode_split_len(int32_t ns, int32_t hkv, int32_t group, int32_t max_ctx);

}  // namespace hswa
