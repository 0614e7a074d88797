// Eviction from the cache by accumulated attention weight: which keys of a
// (sequence, KV head) stay, and their move to the pages that hold them from
// then on.
//
// Selection. The first `sinks` and the last `recent` keys stay; of the others
// the `pick` keys of the highest scores, ties to the lowest position. One
// workgroup per (sequence, KV head) finds the pick-th highest score by its
// digits, from the top (a histogram in LDS per digit), then writes the kept
// positions in order: every wave counts the kept ones of its stretch, and a
// ballot ranks those of 64 positions.
//
// Move. Kept keys keep their order, so slot i of the new pages is the i-th kept
// position; every KV head keeps its own set (a page holds its heads apart). One
// workgroup per 32 slots of a (sequence, KV head).
#include <algorithm>

#include "hswa_common.h"
#include "hswa_launch.h"

namespace hswa {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kDigit = 11;  // bits of a digit: three passes over 32-bit scores
constexpr int kBins = 1 << kDigit;
constexpr int kCopyThreads = 256;
constexpr int kSlots = 32;  // slots of the new pages per workgroup of the move
constexpr int kMaxCopyGrid = 1 << 20;

// What a sequence keeps, by count: its first and last keys and those picked by
// score out of [sinks, len - recent).
struct Keep {
  int len, keep, sinks, recent, pick;
};
__device__ __forceinline__ Keep keep_of(const EvictParams &p, int b) {
  Keep k;
  k.len = max(min(p.ctx_lens[b], p.max_ctx), 0);
  k.keep = max(min(min(p.budgets[b], k.len), p.max_keep), 0);
  k.recent = min(p.num_recent, k.keep);
  k.sinks = min(p.num_sinks, k.keep - k.recent);
  k.pick = k.keep - k.recent - k.sinks;
  return k;
}

// Scores as whole numbers in the same order (the two zeros are equal; a NaN
// counts as -infinity).
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __builtin_bit_cast(uint32_t, s != s ? -INFINITY : s + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t wsum[2][kSelectWaves];
  __shared__ uint32_t found[2];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int b = (int)(blockIdx.x / p.hkv), g = (int)(blockIdx.x - (int64_t)b * p.hkv);
  const Keep n = keep_of(p, b);
  if (g == 0 && tid == 0) p.new_lens[b] = n.keep;
  const int64_t row = (int64_t)b * p.hkv + g;
  const float *scores = p.scores + row * p.score_stride;
  int32_t *kept = p.kept + row * p.max_keep;
  float *out = p.scores_out ? p.scores_out + row * p.out_stride : nullptr;
  auto emit = [&](int slot, int pos) {
    kept[slot] = pos;
    if (out) out[slot] = scores[pos];
  };
  const int lo = n.sinks, hi = n.len - n.recent;
  for (int i = tid; i < n.sinks; i += kSelectThreads) emit(i, i);
  for (int i = tid; i < n.recent; i += kSelectThreads) emit(n.keep - n.recent + i, hi + i);
  if (n.pick == 0) return;
  if (n.pick == hi - lo) {
    for (int i = tid; i < n.pick; i += kSelectThreads) emit(lo + i, lo + i);
    return;
  }
  // The pick-th highest key, digit by digit: `top` is what is known of it, of
  // the keys that share `top` the `need` highest stay.
  uint32_t top = 0, known = 0, need = n.pick;
  bool ties = true;  // whether only some of the keys equal to `top` stay
  for (int shift = 32 - kDigit;; shift = max(shift - kDigit, 0)) {
    const uint32_t digit = known == 0xFFFFFFFFu << (32 - 2 * kDigit) ? (1u << (32 - 2 * kDigit)) - 1 : kBins - 1;
    for (int i = tid; i < kBins; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kSelectThreads) {
      const uint32_t k = score_key(scores[i]);
      if ((k & known) == top) atomicAdd(&hist[(k >> shift) & digit], 1u);
    }
    __syncthreads();
    // the bins from the highest down, two a thread: where the count reaches `need`
    const int hb = kBins - 1 - 2 * tid;
    const uint32_t c0 = hist[hb], c1 = hist[hb - 1];
    uint32_t s = c0 + c1;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const uint32_t t = __shfl_up(s, off, kWave);
      if (lane >= off) s += t;
    }
    if (lane == kWave - 1) wsum[0][wave] = s;
    __syncthreads();
    uint32_t before = s - c0 - c1;
    for (int w = 0; w < wave; ++w) before += wsum[0][w];
    if (before < need && need <= before + c0 + c1) {
      const bool first = need <= before + c0;
      found[0] = first ? hb : hb - 1;
      found[1] = first ? before : before + c0;
    }
    __syncthreads();
    const uint32_t d = found[0];
    need -= found[1];
    top |= d << shift;
    known |= digit << shift;
    ties = hist[d] > need;
    __syncthreads();  // (hist, wsum and found are written again)
    if (shift == 0 || !ties) break;
  }
  // Kept: keys above `top`, and of those equal to it (in its known digits) all,
  // or the first `need` by position.
  const int stretch = ((hi - lo + kSelectWaves * kWave - 1) / (kSelectWaves * kWave)) * kWave;
  const int w0 = min(hi, lo + wave * stretch), w1 = min(hi, w0 + stretch);
  uint32_t above = 0, equal = 0;
  for (int i0 = w0; i0 < w1; i0 += kWave) {
    const int i = i0 + lane;
    const uint32_t k = i < w1 ? score_key(scores[i]) & known : 0;
    above += __popcll(__ballot(i < w1 && k > top));
    equal += __popcll(__ballot(i < w1 && k == top));
  }
  if (lane == 0) {
    wsum[0][wave] = above;
    wsum[1][wave] = equal;
  }
  __syncthreads();
  uint32_t slot = 0, eq = 0;
  for (int w = 0; w < wave; ++w) {
    slot += wsum[0][w];
    eq += wsum[1][w];
  }
  if (!ties) need = 0xFFFFFFFFu;
  slot += n.sinks + min(eq, need);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int i0 = w0; i0 < w1; i0 += kWave) {
    const int i = i0 + lane;
    const uint32_t k = i < w1 ? score_key(scores[i]) & known : 0;
    const uint64_t same = __ballot(i < w1 && k == top);
    const bool keep = i < w1 && (k > top || (k == top && eq + __popcll(same & below) < need));
    const uint64_t mine = __ballot(keep);
    if (keep) emit((int)slot + __popcll(mine & below), i);
    slot += __popcll(mine);
    eq += __popcll(same);
  }
}

// Page of position j of sequence b, -1 if the table has none.
__device__ __forceinline__ int64_t page_of(const PoolView &pv, int b, int j) {
  const int lp = j >> pv.pg_shift;
  if (lp >= pv.stride) return -1;
  const int64_t v = pv.table[(int64_t)b * pv.stride + lp];
  return v >= 0 && v < pv.num_pages ? v : -1;
}

__global__ __launch_bounds__(kCopyThreads) void evict_move_kernel(EvictParams p) {
  __shared__ int64_t from[kSlots];  // element offset of each key's page-head and its offset in the page, -1: none
  __shared__ int off[kSlots];
  const int tid = threadIdx.x;
  const int64_t chunks = (p.max_keep + kSlots - 1) / kSlots, total = chunks * p.ns * p.hkv;
  const int pgm = (1 << p.src.pg_shift) - 1;
  for (int64_t item = blockIdx.x; item < total; item += gridDim.x) {
    const int64_t row = item / chunks;
    const int b = (int)(row / p.hkv), g = (int)(row - (int64_t)b * p.hkv);
    const int s0 = (int)(item - row * chunks) * kSlots;
    const int n = min(keep_of(p, b).keep - s0, kSlots);  // slots of this workgroup
    if (n <= 0) continue;  // (the same for every thread)
    __syncthreads();
    if (tid < kSlots) {
      const int j = tid < n ? p.kept[row * p.max_keep + s0 + tid] : 0;
      from[tid] = tid < n ? page_of(p.src, b, j) : -1;
      off[tid] = j & pgm;
    }
    __syncthreads();
    // K: 16-byte pieces in the order of the new block, so that stores are whole runs
    const int rb = p.dst.vb_shift - 1;  // log2 of the rows of a half block
    for (int x = tid; x < kSlots * 16; x += kCopyThreads) {
      const int r = x & ((1 << rb) - 1), piece = (x >> rb) & 3, slab = (x >> (rb + 2)) & 3, half = (x >> (rb + 4)) & 1;
      const int i = ((x >> (rb + 5)) << (rb + 1)) + 8 * (r >> 2) + 4 * half + (r & 3);
      const int d = 32 * slab + 8 * piece;
      const int64_t to = page_of(p.dst, b, s0 + i);
      if (i < n && to >= 0) {
        const u32x4 z = {0u, 0u, 0u, 0u};
        const u32x4 v = from[i] >= 0 ? ldg128(p.src.k_pool + k_offset(p.src, from[i], p.hkv, g, off[i], d)) : z;
        stg128(p.dst.k_pool + k_offset(p.dst, to, p.hkv, g, (s0 + i) & pgm, d), v);
      }
    }
    // V: eight slots of one dim a thread
    for (int x = tid; x < kSlots * 16; x += kCopyThreads) {
      const int i0 = 8 * (x & 3), d = x >> 2;
      const int64_t to = page_of(p.dst, b, s0 + i0);
      if (i0 >= n || to < 0) continue;
      uint16_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = i0 + e < n && from[i0 + e] >= 0 ? p.src.v_pool[v_offset(p.src, from[i0 + e], p.hkv, g, off[i0 + e], d)] : 0;
      uint16_t *dst = p.dst.v_pool + v_offset(p.dst, to, p.hkv, g, (s0 + i0) & pgm, d);
      if (i0 + 8 <= n) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = v[2 * j] | (uint32_t)v[2 * j + 1] << 16;
        stg128(dst, w);
      } else {
        for (int e = 0; i0 + e < n; ++e) dst[e] = v[e];
      }
    }
  }
}

}  // namespace

hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream) {
  const hipError_t e = launch_kernel(evict_select_kernel, dim3((unsigned)(p.ns * p.hkv)), dim3(kSelectThreads), stream, p);
  if (e != hipSuccess) return e;
  const int64_t items = (int64_t)((p.max_keep + kSlots - 1) / kSlots) * p.ns * p.hkv;
  return launch_kernel(evict_move_kernel, dim3((unsigned)std::min<int64_t>(items, kMaxCopyGrid)), dim3(kCopyThreads),
                       stream, p);
}

}  // namespace hswa
