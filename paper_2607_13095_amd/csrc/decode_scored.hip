// Decode that also adds up what attention every key gets: the weight of key j
// in KV head g is the sum over the call's queries and g's query heads h of
//     exp2(scale log2(e) <q_h, k_j> - lse_h),
// lse_h the row's log2 sum-exp over all its keys. That is known only once the
// whole context has been read, so there are three kernels: the split decode
// (decode_kernels.h, row sums in fp32), the merge of its partials, which also
// leaves the rows' log-sum-exps, and the weights, which read K a second time and
// form the scores anew on the matrix cores.
#include "decode_kernels.h"

namespace hswa {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kWaveChunks = 4;  // 32-key chunks a wave holds at once
constexpr int kScoreKeys = kScoreThreads / kWave * kWaveChunks * kChunk;  // keys of a workgroup

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

// Weights of 512 keys of a (sequence, KV head), 128 a wave. kOnePage: a
// 32-key chunk lies in one page.
template <bool kOnePage>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ScoredParams sp) {
  const DecodeParams &p = sp.d;
  const PoolView &pv = p.pool;
  const int lane = threadIdx.x & (kWave - 1), wave = uni((int)(threadIdx.x / kWave));
  const int r = lane & 15, q = lane >> 4;
  const int tiles = (p.max_ctx + kScoreKeys - 1) / kScoreKeys;
  const int64_t rows = (int64_t)p.ns * p.hkv;
  const int64_t bg = blockIdx.x % rows;
  const int tile = (int)(blockIdx.x / rows);
  const int b = (int)(bg / p.hkv), g = (int)(bg - (int64_t)b * p.hkv);
  const int ctx = min(p.ctx_lens[b], p.max_ctx);
  const int k0 = tile * kScoreKeys + wave * kWaveChunks * kChunk;  // this wave's first key
  if (tile >= tiles || k0 >= ctx) return;
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
  for (int c0 = 0; c0 < ncols; c0 += kCols) {
    const int col = c0 + r;
    const bool valid = col < ncols;
    const int qi = valid ? col / p.group : 0;
    const int64_t row = ((int64_t)b * p.nq + qi) * p.hq + (int64_t)g * p.group + (valid ? col - qi * p.group : 0);
    const float lse = valid ? p.row_lse[row] : INFINITY;
    const int last = pos0 + qi;  // the last key the column sees
    u32x4 qf[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) qf[t] = ldg128(p.q + row * kHeadDim + 32 * t + 8 * q);
#pragma unroll
    for (int c = 0; c < kWaveChunks; ++c) {
      f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = sa;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        sa = mfma16x16x32(ka[c][t], qf[t], sa);
        sb = mfma16x16x32(kb[c][t], qf[t], sb);
      }
      const int j0 = k0 + c * kChunk + 8 * q;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float s = i < 4 ? sa[i & 3] : sb[i & 3];
        const float e = fast_exp2(fmaf(s, p.scale_log2, -lse));
        w[c][i] += valid && held[c] && j0 + i <= last ? e : 0.f;
      }
    }
  }
#pragma unroll
  for (int c = 0; c < kWaveChunks; ++c) {
    float mine = 0.f;  // lane r of a row takes key 8 q + r (r < 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = row_sum16(w[c][i]);
      mine = r == i ? t : mine;
    }
    const int j = k0 + c * kChunk + 8 * q + r;
    if (r < 8 && j < ctx) {
      const int64_t at = bg * sp.stride + j;
      sp.scores_out[at] = (sp.scores_in ? sp.scores_in[at] : 0.f) + mine;
    }
  }
}

template <int kCGd>
hipError_t launch_cg(const ScoredParams &p0, hipStream_t stream) {
  ScoredParams sp = p0;
  DecodeParams &p = sp.d;
  p.item_cols = kCols * kCGd;
  const bool one_page = p.pool.pg_shift >= 5;
  hipError_t e = one_page ? resident_split_waves<true, kCGd, kScored>(p.span_waves)
                          : resident_split_waves<false, kCGd, kScored>(p.span_waves);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(p.span_waves / kWaves)), block(kWave * kWaves);
  e = one_page ? launch_kernel(decode_kernel<true, true, kCGd, kScored>, grid, block, stream, p)
               : launch_kernel(decode_kernel<true, false, kCGd, kScored>, grid, block, stream, p);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)p.ns * p.nq * p.hq;
  constexpr int per_block = kMergeThreads / kWave;
  e = rows <= kWideMergeRows
          ? launch_kernel(decode_merge_kernel<per_block, kScored>, dim3((unsigned)rows), dim3(kMergeThreads), stream, p)
          : launch_kernel(decode_merge_kernel<1, kScored>, dim3((unsigned)((rows + per_block - 1) / per_block)),
                          dim3(kMergeThreads), stream, p);
  if (e != hipSuccess) return e;
  const int64_t items = (int64_t)p.ns * p.hkv * ((p.max_ctx + kScoreKeys - 1) / kScoreKeys);
  return one_page ? launch_kernel(score_kernel<true>, dim3((unsigned)items), dim3(kScoreThreads), stream, sp)
                  : launch_kernel(score_kernel<false>, dim3((unsigned)items), dim3(kScoreThreads), stream, sp);
}

}  // namespace

hipError_t launch_decode_scored(const ScoredParams &p, hipStream_t stream) {
  return p.d.nq * p.d.group > kCols ? launch_cg<2>(p, stream) : launch_cg<1>(p, stream);
}

}  // namespace hswa
