// Decode that also adds up what attention every key gets: the weight of key j
// in KV head g is the sum over the call's queries and g's query heads h of
//     exp2(scale log2(e) <q_h, k_j> - lse_h),
// lse_h the row's log2 sum-exp over all its keys. That is known only once the
// whole context has been read, so the weights come after the split decode
// (decode_kernels.h, row sums in fp32), in one of two ways:
//   up to kKeepColumns columns (queries x heads of a KV head): the decode also
//     stores the scores in fp32, and one more kernel merges the rows and turns
//     the scores into weights. A column costs 8 bytes a key (written and read),
//     a key's K and V 512.
//   more: the attention is that of decode_shared.hip, every sequence a group of
//     its own (its queries see all of its keys but the last alike), which reads
//     the keys once for 256 columns where the split decode does for 32; its merge
//     leaves the rows' log-sum-exps, and another kernel reads K a second time
//     (256 bytes a key, whatever the columns) and forms the scores anew on the
//     matrix cores. (16 queries, 32 / 8 heads, 4 x 3000 - 9000, PG 16: 41 us by
//     the split decode, 27 so.)
#include <algorithm>
#include <type_traits>

#include "decode_kernels.h"

namespace hswa {
namespace {

constexpr int kScoreThreads = kMergeThreads;
constexpr int kKeptKeys = 4 * kScoreThreads;  // keys of a workgroup, from kept scores
constexpr int kMaxScoreGrid = 1 << 20;
constexpr int score_keys(int wave_chunks) { return kScoreThreads / kWave * wave_chunks * kChunk; }  // of a workgroup
// Below this many workgroups of 512 keys (1.5 a compute unit) they take 128 each. us
// a call with 128 and 512, 64 / 8 heads: 1 x 1000, 4 queries 24.0 and 26.1; 1 x
// 4000, 16 queries 30.6 and 36.4; 8 / 1, 24 x 300 - 6000, 4 queries 32.2 and 33.6;
// with more, 32 / 8, 4 x 3000 - 9000, 16 queries 53.9 and 46.5 (each reads all of
// the queries).
constexpr int kFewItems = 384;

// Sum over the 16 lanes of a row.
__device__ __forceinline__ float row_sum16(float x) {
#define HSWA_ROW_ADD(ctrl)                                                                              \
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, 0xf, 0xf, false))
  HSWA_ROW_ADD(0x128);  // rotate the row by 8, 4, 2, 1
  HSWA_ROW_ADD(0x124);
  HSWA_ROW_ADD(0x122);
  HSWA_ROW_ADD(0x121);
#undef HSWA_ROW_ADD
  return x;
}

// Weights of the keys of a (sequence, KV head), kWaveChunks 32-key chunks a wave.
// kOnePage: a chunk lies in one page.
template <bool kOnePage, int kWaveChunks>
__global__ __launch_bounds__(kScoreThreads) __attribute__((amdgpu_waves_per_eu(kWaveChunks == 1 ? 4 : 2)))
void score_kernel(ScoredParams sp) {
  constexpr int kScoreKeys = score_keys(kWaveChunks);
  const DecodeParams &p = sp.s.d;
  const PoolView &pv = p.pool;
  const int lane = threadIdx.x & (kWave - 1), wave = uni((int)(threadIdx.x / kWave));
  const int r = lane & 15, q = lane >> 4;
  const int64_t rows = (int64_t)p.ns * p.hkv, items = rows * ((p.max_ctx + kScoreKeys - 1) / kScoreKeys);
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t bg = item % rows;
    const int tile = (int)(item / rows);
    const int b = (int)(bg / p.hkv), g = (int)(bg - (int64_t)b * p.hkv);
    const int ctx = min(p.ctx_lens[b], p.max_ctx);
    const int k0 = tile * kScoreKeys + wave * kWaveChunks * kChunk;  // this wave's first key
    if (k0 >= ctx) continue;
    const int pos0 = ctx - p.nq;  // the first query's position
    const int ncols = p.nq * p.group;

    u32x4 ka[kWaveChunks][4], kb[kWaveChunks][4];
    bool held[kWaveChunks];  // whether this lane's keys 8 q .. 8 q + 7 of the chunk are in the pool
#pragma unroll
    for (int c = 0; c < kWaveChunks; ++c) {
      const int key = k0 + c * kChunk;
      auto page_of = [&](int k) {
        const int lp = k >> pv.pg_shift;
        if (k >= ctx) return -1;  // (a page past the context is not read)
        const int64_t v = pv.table[(int64_t)b * pv.stride + lp];
        return v >= 0 && v < pv.num_pages ? (int)v : -1;
      };
      const int pa = page_of(key), pb = kOnePage ? pa : page_of(key + 16);
      held[c] = (kOnePage || !(q & 2) ? pa : pb) >= 0;
      const int page = kOnePage || !(r & 8) ? pa : pb;  // of this lane's K rows
      const char *base = reinterpret_cast<const char *>(pv.k_pool) +
                         (((int64_t)max(page, 0) * p.hkv + g) << (pv.pg_shift + kHeadDimShift + 1));
      uint32_t off;
      if constexpr (kOnePage) off = ((key & ((1 << pv.pg_shift) - 1)) << (kHeadDimShift + 1)) + lane * 16;
      else off = (q * 8 + (r & 7)) * 16;
      constexpr uint32_t slab = kOnePage ? 1024 : 512;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 z = {0u, 0u, 0u, 0u};
        ka[c][t] = page >= 0 ? ldg128(base + off + slab * t) : z;
        kb[c][t] = page >= 0 ? ldg128(base + off + slab * (t + 4)) : z;
      }
    }
    float w[kWaveChunks][8] = {};  // keys 8 q + i of the chunk, column r's share
    // column r of a group of 16: its queries' operands and log-sum-exp, loaded a group ahead
    struct Columns {
      u32x4 q[4];
      float lse;
      int last;  // the last key it sees
    };
    auto load_columns = [&](int c0, Columns &x) {
      const int col = c0 + r;
      const bool valid = col < ncols;
      const int qi = valid ? col / p.group : 0;
      const int64_t row = ((int64_t)b * p.nq + qi) * p.hq + (int64_t)g * p.group + (valid ? col - qi * p.group : 0);
      x.lse = valid ? p.row_lse[row] : INFINITY;  // (weight 0)
      x.last = pos0 + qi;
#pragma unroll
      for (int t = 0; t < 4; ++t) x.q[t] = ldg128(p.q + row * kHeadDim + 32 * t + 8 * q);
    };
    Columns next;
    load_columns(0, next);
    // kMasked: some column does not see all of the wave's keys
    auto columns = [&](auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      for (int c0 = 0; c0 < ncols; c0 += kCols) {
        const Columns now = next;
        if (c0 + kCols < ncols) load_columns(c0 + kCols, next);
#pragma unroll
        for (int c = 0; c < kWaveChunks; ++c) {
          f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = sa;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            sa = mfma16x16x32(ka[c][t], now.q[t], sa);
            sb = mfma16x16x32(kb[c][t], now.q[t], sb);
          }
          const int j0 = k0 + c * kChunk + 8 * q;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float s = i < 4 ? sa[i & 3] : sb[i & 3];
            const float e = fast_exp2(fmaf(s, p.scale_log2, -now.lse));
            w[c][i] += !kMasked || j0 + i <= now.last ? e : 0.f;
          }
        }
      }
    };
    if (k0 + kWaveChunks * kChunk - 1 <= pos0) columns(std::false_type{});
    else columns(std::true_type{});
#pragma unroll
    for (int c = 0; c < kWaveChunks; ++c) {
      float mine = 0.f;  // lane r of a row takes key 8 q + r (r < 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = row_sum16(w[c][i]);
        mine = r == i ? t : mine;
      }
      if (!held[c]) mine = 0.f;
      const int j = k0 + c * kChunk + 8 * q + r;
      if (r < 8 && j < ctx) {
        const int64_t at = bg * sp.stride + j;
        sp.scores_out[at] = (sp.scores_in ? sp.scores_in[at] : 0.f) + mine;
      }
    }
  }
}

// The rows' merge (the first `merge_blocks` workgroups), and the weights of 1024
// keys of a (sequence, KV head) from the scores that the decode stored, four
// keys a thread.
template <int kRowWaves>
__global__ __launch_bounds__(kScoreThreads) void scored_finish_kernel(ScoredParams sp) {
  const DecodeParams &p = sp.s.d;
  if (blockIdx.x < (unsigned)sp.merge_blocks) {
    merge_rows<kRowWaves, kKept>(p, blockIdx.x);
    return;
  }
  __shared__ float s_lse[kKeepColumns];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = uni((int)(tid / kWave));
  const int ncols = p.nq * p.group;
  int64_t total = 0;  // chunks of all sequences: the spans' length (as in the decode kernel)
  for (int s0 = 0; s0 < p.ns; s0 += kWave) total += wave_sum64(seq_chunks(p, s0 + lane));
  total = uni64(total) * p.hkv;
  const int64_t per = max((int64_t)(p.split_len / kChunk), (total + p.span_waves - 1) / p.span_waves);
  const int64_t rows = (int64_t)p.ns * p.hkv, items = rows * ((p.max_ctx + kKeptKeys - 1) / kKeptKeys);
  // whether four keys' scores are one 16-byte access in every row
  const bool aligned = ((reinterpret_cast<uintptr_t>(sp.scores_in) | reinterpret_cast<uintptr_t>(sp.scores_out) |
                         (uintptr_t)(sp.stride * sizeof(float))) & 15) == 0;
  const int64_t step = (int64_t)gridDim.x - sp.merge_blocks;
  for (int64_t item = (int64_t)blockIdx.x - sp.merge_blocks; item < items; item += step) {
    const int64_t bg = item % rows;
    const int b = (int)(bg / p.hkv), g = (int)(bg - (int64_t)b * p.hkv);
    const int ctx = min(p.ctx_lens[b], p.max_ctx);
    const int k0 = (int)(item / rows) * kKeptKeys;
    if (k0 >= ctx) continue;  // (the same for every thread)
    const int j = k0 + 4 * tid;
    const int64_t at = bg * sp.stride + j;
    f32x4 old = {0.f, 0.f, 0.f, 0.f};  // (its loads go out before the others)
    if (sp.scores_in) {
      if (aligned && j + 3 < ctx) {
        old = *reinterpret_cast<const f32x4 *>(sp.scores_in + at);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j + i < ctx) old[i] = sp.scores_in[at + i];
      }
    }
    int64_t before = 0;
    for (int s0 = 0; s0 < b; s0 += kWave) before += wave_sum64(s0 + lane < b ? seq_chunks(p, s0 + lane) : 0);
    const int nch = (ctx + kChunk - 1) / kChunk;
    const int64_t seg = uni64(before) * p.hkv + (int64_t)g * nch;
    const int pieces = (int)((seg + nch - 1) / per - seg / per) + 1;
    __syncthreads();  // (s_lse of the item before has been read)
    // the columns' log-sum-exps: four a wave (kKeepColumns = 16), their loads together
    constexpr int kEach = kKeepColumns / (kScoreThreads / kWave);
    const float *lse[kEach];
    float first[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int c = min(wave + e * (kScoreThreads / kWave), ncols - 1), qi = c / p.group;
      lse[e] = p.ws_lse + (((int64_t)b * p.nq + qi) * p.hq + (int64_t)g * p.group + (c - qi * p.group)) * p.max_splits;
      first[e] = lane < pieces ? lse[e][lane] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const auto most = [](float a, float b) { return fmaxf(a, b); };
      const auto add = [](float a, float b) { return a + b; };
      float mx = first[e];
      for (int s = lane + kWave; s < pieces; s += kWave) mx = fmaxf(mx, lse[e][s]);
      mx = last_lane(wave_scan(mx, -INFINITY, most));
      // (a row that sees no key has scores of -infinity: weight 0 under any finite or +infinite sum)
      const float base = mx == -INFINITY ? 0.f : mx;
      float sum = fast_exp2(first[e] - base);
      for (int s = lane + kWave; s < pieces; s += kWave) sum += fast_exp2(lse[e][s] - base);
      sum = last_lane(wave_scan(sum, 0.f, add));
      const int c = wave + e * (kScoreThreads / kWave);
      if (lane == 0 && c < ncols) s_lse[c] = mx == -INFINITY ? INFINITY : mx + __log2f(sum);
    }
    __syncthreads();
    if (j < ctx) {
      const f32x4 *src = reinterpret_cast<const f32x4 *>(p.ws_s) + (bg * p.max_chunks + (j >> 5)) * ncols * 8 +
                         ((j & (kChunk - 1)) >> 2);
      f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int c = 0; c < ncols; ++c) {
        const f32x4 s = src[8 * c];
        const float l = s_lse[c];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] += fast_exp2(s[i] - l);
      }
      if (aligned && j + 3 < ctx) {
        *reinterpret_cast<f32x4 *>(sp.scores_out + at) = old + w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j + i < ctx) sp.scores_out[at + i] = old[i] + w[i];
      }
    }
  }
}

hipError_t launch_kept(const ScoredParams &p0, hipStream_t stream) {
  constexpr int kCGd = 1;
  static_assert(kKeepColumns <= kCGd * kCols, "one column item per KV head");
  ScoredParams sp = p0;
  DecodeParams &p = sp.s.d;
  p.item_cols = kCols * kCGd;
  const bool one_page = p.pool.pg_shift >= 5;
  hipError_t e = one_page ? resident_split_waves<true, kCGd, kKept>(p.span_waves)
                          : resident_split_waves<false, kCGd, kKept>(p.span_waves);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(p.span_waves / kWaves)), block(kWave * kWaves), threads(kScoreThreads);
  e = one_page ? launch_kernel(decode_kernel<true, true, kCGd, kKept>, grid, block, stream, p)
               : launch_kernel(decode_kernel<true, false, kCGd, kKept>, grid, block, stream, p);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)p.ns * p.nq * p.hq;
  constexpr int per_block = kMergeThreads / kWave;
  const bool wide = rows <= kWideMergeRows;
  sp.merge_blocks = wide ? rows : (rows + per_block - 1) / per_block;
  const int64_t items = (int64_t)p.ns * p.hkv * ((p.max_ctx + kKeptKeys - 1) / kKeptKeys);
  const dim3 both((unsigned)(sp.merge_blocks + std::min<int64_t>(items, kMaxScoreGrid)));
  return wide ? launch_kernel(scored_finish_kernel<per_block>, both, threads, stream, sp)
              : launch_kernel(scored_finish_kernel<1>, both, threads, stream, sp);
}

template <int kWaveChunks>
hipError_t launch_scores(const ScoredParams &p, hipStream_t stream) {
  const DecodeParams &d = p.s.d;
  constexpr int keys = score_keys(kWaveChunks);
  const int64_t items = (int64_t)d.ns * d.hkv * ((d.max_ctx + keys - 1) / keys);
  const dim3 grid((unsigned)std::min<int64_t>(items, kMaxScoreGrid)), threads(kScoreThreads);
  return d.pool.pg_shift >= 5 ? launch_kernel(score_kernel<true, kWaveChunks>, grid, threads, stream, p)
                              : launch_kernel(score_kernel<false, kWaveChunks>, grid, threads, stream, p);
}

}  // namespace

hipError_t launch_decode_scored(const ScoredParams &p, hipStream_t stream) {
  const DecodeParams &d = p.s.d;
  if (d.nq * d.group <= kKeepColumns) return launch_kept(p, stream);
  const hipError_t e = launch_decode_shared_scored(p.s, stream);
  if (e != hipSuccess) return e;
  const int64_t items = (int64_t)d.ns * d.hkv * ((d.max_ctx + score_keys(4) - 1) / score_keys(4));
  return items < kFewItems ? launch_scores<1>(p, stream) : launch_scores<4>(p, stream);
}

}  // namespace hswa
