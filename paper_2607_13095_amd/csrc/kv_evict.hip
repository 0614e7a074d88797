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
// workgroup per 32 slots of a (sequence, KV head). Where these are no more than
// the compute units, one kernel does both.
#include <algorithm>

#include "hswa_common.h"
#include "hswa_launch.h"

namespace hswa {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kDigit = 11;  // bits of a digit: three passes over 32-bit scores
constexpr int kBins = 1 << kDigit;
constexpr int kBatch = 16;
constexpr int kListed = 512;  // keys of a wave's list
constexpr int kCopies = 4;  // of the histogram, for lanes that meet in a bin
constexpr int kMoveThreads = 256;
constexpr int kSlots = 32;        // slots of the new pages per workgroup of the move
constexpr int kMaxMoveGrid = 1 << 20;
constexpr int kSmallItems = 256;  // a workgroup per compute unit

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
  const uint32_t u = __builtin_bit_cast(uint32_t, fmaxf(s + 0.f, -INFINITY));
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// kPer: scores that a thread holds in registers, 64 positions of a wave apart; 0:
// any number, read again for each pass, kBatch loads at a time (one at a time a
// pass over 58K scores took 20 us; 64 held spilled). The second pass lists the keys
// that share the first digit sought (a twentieth of them, if the scores spread over
// some orders of magnitude), for the third digit and the counts: three passes
// instead of five, unless a wave's list is too short (8 x 58K, 8 KV heads: 54 us of
// selection and 48; 2 x 130K to 2000: 164 us a call and 138).
template <int kPer>
struct SelectLds {
  alignas(16) uint32_t hist[kBins * kCopies];  // (16-byte reads)
  uint32_t wsum[2][kSelectWaves];
  uint32_t found[3];
  uint32_t over;                                         // (kPer 0) whether a wave's list is too short
  uint32_t list[kSelectWaves][kPer == 0 ? kListed : 1];  // keys of the first digit sought, in order
};
// emit(slot, position, score) for every kept key of row (b, g), by kSelectThreads.
template <int kPer, typename Emit>
__device__ __forceinline__ void select_row(const Keep &n, const float *scores, SelectLds<kPer> &lds, Emit emit) {
  constexpr int kEach = kBins / kSelectThreads;  // bins of a thread
  auto &hist = lds.hist;
  auto &wsum = lds.wsum;
  auto &found = lds.found;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lo = n.sinks, hi = n.len - n.recent;
  // this wave's stretch of the positions that are picked from: groups of 64
  const int groups = (hi - lo + kSelectWaves * kWave - 1) / (kSelectWaves * kWave);
  const int w0 = min(hi, lo + wave * groups * kWave), w1 = min(hi, w0 + groups * kWave);
  float held[kPer > 0 ? kPer : 1];
  const bool choose = n.pick > 0 && n.pick < hi - lo;
  if (kPer > 0 && choose) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = w0 + e * kWave + lane;
      held[e] = i < w1 ? scores[i] : 0.f;
    }
  }
  for (int i = tid; i < n.sinks; i += kSelectThreads) emit(i, i, scores[i]);
  for (int i = tid; i < n.recent; i += kSelectThreads) emit(n.keep - n.recent + i, hi + i, scores[hi + i]);
  if (!choose) {
    for (int i = tid; i < n.pick; i += kSelectThreads) emit(lo + i, lo + i, scores[lo + i]);
    return;
  }
  // f(position, key, whether there is one) for 64 positions of the stretch at a time
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (kPer > 0) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        if (w0 + e * kWave >= w1) break;  // (the same for the wave)
        const int i = w0 + e * kWave + lane;
        f(i, score_key(held[e]), held[e], i < w1);
      }
    } else {
      // the next batch's loads go out before this one is worked on; whole batches
      // need no bounds
      auto load = [&](int i0, float (&s)[kBatch]) {
#pragma unroll
        for (int e = 0; e < kBatch; ++e) {
          const int i = i0 + e * kWave + lane;
          s[e] = i < w1 ? scores[i] : 0.f;
        }
      };
      float next[kBatch];
      load(w0, next);
      for (int i0 = w0; i0 < w1; i0 += kBatch * kWave) {
        float s[kBatch];
#pragma unroll
        for (int e = 0; e < kBatch; ++e) s[e] = next[e];
        load(i0 + kBatch * kWave, next);
        if (i0 + kBatch * kWave <= w1) {
#pragma unroll
          for (int e = 0; e < kBatch; ++e) f(i0 + e * kWave + lane, score_key(s[e]), s[e], true);
        } else {
#pragma unroll
          for (int e = 0; e < kBatch; ++e) {
            if (i0 + e * kWave >= w1) break;
            const int i = i0 + e * kWave + lane;
            f(i, score_key(s[e]), s[e], i < w1);
          }
        }
      }
    }
  };
  // The pick-th highest key, digit by digit: `top` is what is known of it, of
  // the keys that share `top` the `need` highest stay.
  uint32_t top = 0, known = 0, need = n.pick;
  bool ties = true;  // whether only some of the keys equal to `top` stay
  uint32_t higher = 0;  // (kPer 0) this wave's keys of a higher first digit
  int listed = 0;       // and those of its list
  if (tid == 0) lds.over = 0;
#pragma unroll 1
  for (int shift = 32 - kDigit;; shift = max(shift - kDigit, 0)) {
    const uint32_t digit = shift == 0 ? (1u << (32 - 2 * kDigit)) - 1 : kBins - 1;
    for (int i = tid; i < kBins * kCopies; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    auto count_digit = [&](uint32_t k) {
      atomicAdd(&hist[((k >> shift) & digit) * kCopies + (lane & (kCopies - 1))], 1u);
    };
    if (kPer == 0 && shift == 32 - 2 * kDigit) {
      each([&](int, uint32_t k, float, bool in) {
        const uint64_t same = __ballot(in && (k & known) == top);
        higher += __popcll(__ballot(in && (k & known) > top));
        if (same == 0) return;
        if ((same >> lane) & 1) {
          const int at = listed + __popcll(same & (((uint64_t)1 << lane) - 1));
          if (at < kListed) lds.list[wave][at] = k;
          count_digit(k);
        }
        listed += __popcll(same);
      });
      if (listed > kListed && lane == 0) lds.over = 1;  // (cleared before the passes)
    } else if (kPer == 0 && shift == 0 && !lds.over) {
      for (int i = lane; i < listed; i += kWave) {
        const uint32_t k = lds.list[wave][i];
        if ((k & known) == top) count_digit(k);
      }
    } else {
      each([&](int, uint32_t k, float, bool in) {
        if (in && (k & known) == top) count_digit(k);
      });
    }
    __syncthreads();
    // the bins from the highest down, kEach a thread: where the count reaches `need`
    const int hb = kBins - 1 - kEach * tid;
    uint32_t count[kEach], s = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      count[e] = 0;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) count[e] += hist[(hb - e) * kCopies + c];
      s += count[e];
    }
    const uint32_t mine = s;
    s = wave_scan(s, 0u, [](uint32_t a, uint32_t b) { return a + b; });
    if (lane == kWave - 1) wsum[0][wave] = s;
    __syncthreads();
    uint32_t before = s - mine;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) before += w < wave ? wsum[0][w] : 0u;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      if (before < need && need <= before + count[e]) {
        found[0] = hb - e;
        found[1] = before;
        found[2] = count[e];
      }
      before += count[e];
    }
    __syncthreads();
    need -= found[1];
    top |= found[0] << shift;
    known |= digit << shift;
    ties = found[2] > need;
    if (shift == 0 || !ties) break;  // (hist is cleared before found is written again, a barrier later)
  }
  // Kept: keys above `top`, and of those equal to it (in its known digits) all,
  // or the first `need` by position.
  uint32_t above = 0, equal = 0;
  const bool by_list = kPer == 0 && (known << kDigit) != 0 && !lds.over;  // (two digits or more are known)
  if (by_list) {
    above = higher;
    for (int i0 = 0; i0 < listed; i0 += kWave) {
      const bool in = i0 + lane < listed;
      const uint32_t k = in ? lds.list[wave][i0 + lane] & known : 0;
      above += __popcll(__ballot(in && k > top));
      equal += __popcll(__ballot(in && k == top));
    }
  } else {
    each([&](int, uint32_t key, float, bool in) {
      const uint32_t k = key & known;
      above += __popcll(__ballot(in && k > top));
      equal += __popcll(__ballot(in && k == top));
    });
  }
  __syncthreads();  // (wsum has been read)
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
  each([&](int i, uint32_t key, float score, bool in) {
    const uint32_t k = key & known;
    const uint64_t same = __ballot(in && k == top);
    const bool keep = in && (k > top || (k == top && eq + __popcll(same & below) < need));
    const uint64_t mine = __ballot(keep);
    if (keep) emit((int)slot + __popcll(mine & below), i, score);
    slot += __popcll(mine);
    eq += __popcll(same);
  });
}

// Where a row's kept positions and their scores go.
struct KeptRow {
  int32_t *kept;
  float *scores;
};
__device__ __forceinline__ KeptRow kept_row(const EvictParams &p, int64_t row) {
  return KeptRow{p.kept + row * p.max_keep, p.scores_out ? p.scores_out + row * p.out_stride : nullptr};
}

template <int kPer>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictParams p) {
  __shared__ SelectLds<kPer> lds;
  const int b = (int)(blockIdx.x / p.hkv), g = (int)(blockIdx.x - (int64_t)b * p.hkv);
  const Keep n = keep_of(p, b);
  if (g == 0 && threadIdx.x == 0) p.new_lens[b] = n.keep;
  const int64_t row = (int64_t)b * p.hkv + g;
  const KeptRow out = kept_row(p, row);
  select_row<kPer>(n, p.scores + row * p.score_stride, lds, [&](int slot, int pos, float score) {
    out.kept[slot] = pos;
    if (out.scores) out.scores[slot] = score;
  });
}

// Page of position j of sequence b, -1 if the table has none.
__device__ __forceinline__ int page_of(const PoolView &pv, int b, int j) {
  const int lp = j >> pv.pg_shift;
  if (lp >= pv.stride) return -1;
  const int64_t v = pv.table[(int64_t)b * pv.stride + lp];
  return v >= 0 && v < pv.num_pages ? (int)v : -1;
}

// 32 slots of the new pages. K moves in 16-byte pieces (8 dims of a key). V is
// stored with a block's keys side by side, so a kept key is 2 bytes here and
// there: each of kVWaves waves takes its share of the dims, loads whole rows of
// the blocks that hold kept keys (kStageBlocks, a power of two, at a time, in
// LDS) and picks from them the slots of each lane, of one dim. kB: keys of a block
// (16 for 16-key pages, else 32). kKWaves: waves that move K; V starts with wave
// kVFirst.
template <int kB, int kStageBlocks, int kKWaves, int kVFirst, int kVWaves>
struct Move {
  static constexpr int kDims = kHeadDim / kVWaves;      // dims of a wave
  static constexpr int kRow = 2 * kB / 16;              // 16-byte pieces of a block's row
  static constexpr int kPad = kRow + 1;                 // and of a row in LDS
  static constexpr int kLoads = kDims * kRow / kWave;   // pieces of a block for a lane
  static constexpr int kLanes = kWave / kDims;          // lanes of a dim
  static constexpr int kPick = kSlots / kLanes;         // slots of a lane
  static_assert(kLoads * kWave == kDims * kRow && kPick % 8 == 0, "whole loads, whole 16-byte stores");
  struct Lds {
    u32x4 stage[kVWaves][kStageBlocks][kDims * kPad];
    int page[kSlots], off[kSlots];  // source page (-1: none) and offset of each slot
    int block[kSlots];              // its block, numbered among those of this workgroup
    int first[kSlots + 1];          // first slot of each block
    int to[kSlots];                 // page of each slot (-1: none)
    int blocks, count;
  };

  // By one wave: lane l < count keeps position j, of page `from`, for a slot on page `to`.
  __device__ static __forceinline__ void plan(Lds &s, int pgm, int count, int j, int from, int to) {
    const int lane = threadIdx.x & (kWave - 1);
    const bool in = lane < count;
    const int before = __shfl_up(j, 1, kWave);
    const uint64_t starts = __ballot(in && (lane == 0 || j / kB != before / kB));
    if (lane < kSlots) {
      s.to[lane] = in ? to : -1;
      s.page[lane] = in ? from : -1;
      s.off[lane] = j & pgm;
      const int blk = __popcll(starts & (((uint64_t)2 << lane) - 1)) - 1;
      s.block[lane] = blk;
      if ((starts >> lane) & 1) s.first[blk] = lane;
    }
    if (lane == 0) {
      s.blocks = __popcll(starts);
      s.first[__popcll(starts)] = count;
      s.count = count;
    }
  }

  // The n slots from s0 on of KV head g, as planned.
  __device__ static __forceinline__ void run(const EvictParams &p, Lds &s, int g, int s0, int n) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int pgm = (1 << p.src.pg_shift) - 1;
    const u32x4 z = {0u, 0u, 0u, 0u};
    if (wave < kKWaves) {
      // K: pieces in the order of the new block, so that stores are whole runs
      constexpr int rb = kB == 32 ? 4 : 3;  // log2 of the rows of a half block
#pragma unroll
      for (int y = 0; y < kSlots * 16 / (kKWaves * kWave); ++y) {
        const int x = tid + y * kKWaves * kWave;
        const int r = x & ((1 << rb) - 1), piece = (x >> rb) & 3, slab = (x >> (rb + 2)) & 3, half = (x >> (rb + 4)) & 1;
        const int i = ((x >> (rb + 5)) << (rb + 1)) + 8 * (r >> 2) + 4 * half + (r & 3);
        const int d = 32 * slab + 8 * piece;
        const int to = s.to[i];
        if (to < 0) continue;
        const u32x4 v = s.page[i] >= 0 ? ldg128(p.src.k_pool + k_offset(p.src, s.page[i], p.hkv, g, s.off[i], d)) : z;
        stg128(p.dst.k_pool + k_offset(p.dst, to, p.hkv, g, (s0 + i) & pgm, d), v);
      }
    }
    if (wave < kVFirst || wave >= kVFirst + kVWaves) return;
    // V: lane = (dim, kPick slots)
    const int vw = wave - kVFirst, d = vw * kDims + lane / kLanes, i0 = kPick * (lane & (kLanes - 1));
    uint32_t val[kPick / 2] = {};  // two slots each
    const int blocks = s.blocks;
    for (int b0 = 0; b0 < blocks; b0 += kStageBlocks) {
      u32x4 ld[kStageBlocks][kLoads];
#pragma unroll
      for (int k = 0; k < kStageBlocks; ++k) {
        const int first = s.first[min(b0 + k, blocks - 1)];
        const int page = s.page[first];
        const uint16_t *src = p.src.v_pool + v_offset(p.src, max(page, 0), p.hkv, g, s.off[first] & ~(kB - 1), vw * kDims);
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
          ld[k][l] = b0 + k < blocks && page >= 0 ? ldg128(src + (l * kWave + lane) * 8) : z;
      }
      wave_exchange();  // (the picks from the blocks before are done)
#pragma unroll
      for (int k = 0; k < kStageBlocks; ++k)
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
          const int x = l * kWave + lane;
          s.stage[vw][k][x / kRow * kPad + x % kRow] = ld[k][l];
        }
      wave_exchange();
#pragma unroll
      for (int e = 0; e < kPick; ++e) {
        const int blk = s.block[i0 + e] - b0;
        const uint16_t *rowp =
            reinterpret_cast<const uint16_t *>(&s.stage[vw][blk & (kStageBlocks - 1)][lane / kLanes * kPad]);
        const uint32_t v = rowp[s.off[i0 + e] & (kB - 1)];
        if (blk >= 0 && blk < kStageBlocks) val[e >> 1] |= v << (16 * (e & 1));
      }
      wave_exchange();
    }
    const int to = s.to[i0];
    if (to < 0) return;
    uint16_t *dst = p.dst.v_pool + v_offset(p.dst, to, p.hkv, g, (s0 + i0) & pgm, d);
#pragma unroll
    for (int h = 0; h < kPick / 8; ++h) {
      if (i0 + 8 * h + 8 <= n) {
        stg128(dst + 8 * h, u32x4{val[4 * h], val[4 * h + 1], val[4 * h + 2], val[4 * h + 3]});
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (i0 + 8 * h + e < n) dst[8 * h + e] = (uint16_t)(val[4 * h + (e >> 1)] >> (16 * (e & 1)));
      }
    }
  }
};

template <int kB, int kStageBlocks>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
  constexpr int kMoveWaves = kMoveThreads / kWave;
  using M = Move<kB, kStageBlocks, kMoveWaves, 0, kMoveWaves>;
  __shared__ typename M::Lds s;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t chunks = (p.max_keep + kSlots - 1) / kSlots, total = chunks * p.ns * p.hkv;
  const int pgm = (1 << p.src.pg_shift) - 1;
  for (int64_t item = blockIdx.x; item < total; item += gridDim.x) {
    const int64_t row = item / chunks;
    const int b = (int)(row / p.hkv), g = (int)(row - (int64_t)b * p.hkv);
    const int s0 = (int)(item - row * chunks) * kSlots;
    __syncthreads();  // (the arrays have been read for the item before)
    if (wave == 0) {
      // the loads that need no other go out together: the length, the kept
      // positions (whatever lies behind them), the pages of the new slots
      const int len = p.new_lens[b];
      const int at = s0 + (lane & (kSlots - 1));
      int j = at < p.max_keep ? p.kept[row * p.max_keep + at] : 0;
      const int to = page_of(p.dst, b, at);
      const int count = min(len - s0, kSlots);
      j = lane < count ? j : 0;
      M::plan(s, pgm, count, j, lane < count ? page_of(p.src, b, j) : -1, to);
    }
    __syncthreads();
    if (s.count <= 0) continue;
    M::run(p, s, g, s0, s.count);
  }
}

// Both for few slots: every workgroup selects for its row by itself and moves
// its 32 slots, half of the waves K and half V; the second launch and the way of
// the positions through memory are saved. us a call, one kernel and two (8 KV
// heads): 1 x 1000 to 300 9.7 and 12.7, 1 x 4100 to 1024 13.6 and 16.0, 1 x 16000
// to 1000 25.2 and 29.0, 32 x 300 to 30 14.5 and 18.5; with more workgroups than
// compute units (two in LDS do not fit one) 2 x 4000 to 1000 23.1 and 19.5.
// kPer as above, not 0.
template <int kPer, int kB>
__global__ __launch_bounds__(kSelectThreads) void evict_small_kernel(EvictParams p) {
  using M = Move<kB, 8, kSelectWaves / 2, kSelectWaves / 2, kB == 32 ? 8 : 4>;
  __shared__ SelectLds<kPer> lds;
  __shared__ typename M::Lds s;
  __shared__ int s_kept[kSlots];
  __shared__ int s_pages[kPer * kSelectThreads / kB];  // the row of the source's table
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int chunks = (p.max_keep + kSlots - 1) / kSlots;
  const int row = (int)blockIdx.x / chunks, s0 = ((int)blockIdx.x - row * chunks) * kSlots;
  const int b = row / p.hkv, g = row - b * p.hkv;
  const Keep n = keep_of(p, b);
  if (g == 0 && s0 == 0 && tid == 0) p.new_lens[b] = n.keep;
  const int count = min(n.keep - s0, kSlots);
  if (count <= 0) return;
  const int to = tid < kSlots ? page_of(p.dst, b, s0 + tid) : -1;
  const int pages = (n.len + (1 << p.src.pg_shift) - 1) >> p.src.pg_shift;
  for (int i = tid; i < pages; i += kSelectThreads) s_pages[i] = page_of(p.src, b, i << p.src.pg_shift);
  const KeptRow out = kept_row(p, row);
  select_row<kPer>(n, p.scores + (int64_t)row * p.score_stride, lds, [&](int slot, int pos, float score) {
    if (slot < s0 || slot >= s0 + kSlots) return;
    s_kept[slot - s0] = pos;
    out.kept[slot] = pos;
    if (out.scores) out.scores[slot] = score;
  });
  __syncthreads();
  if (tid < kWave) {
    const int j = lane < count ? s_kept[lane] : 0;
    M::plan(s, (1 << p.src.pg_shift) - 1, count, j, s_pages[j >> p.src.pg_shift], to);
  }
  __syncthreads();
  M::run(p, s, g, s0, count);
}

template <int kPer>
hipError_t launch_small(const EvictParams &p, int64_t items, hipStream_t stream) {
  const dim3 grid((unsigned)items), threads(kSelectThreads);
  return p.src.vb_shift == 4 ? launch_kernel(evict_small_kernel<kPer, 16>, grid, threads, stream, p)
                             : launch_kernel(evict_small_kernel<kPer, 32>, grid, threads, stream, p);
}

template <int kPer>
hipError_t launch_select(const EvictParams &p, hipStream_t stream) {
  return launch_kernel(evict_select_kernel<kPer>, dim3((unsigned)(p.ns * p.hkv)), dim3(kSelectThreads), stream, p);
}

}  // namespace

hipError_t launch_kv_evict(const EvictParams &p, hipStream_t stream) {
  const int64_t items = (int64_t)((p.max_keep + kSlots - 1) / kSlots) * p.ns * p.hkv;
  // Scores in registers as far as they fit: us a call with 8, 16, 32 of them and by
  // passes, 1 x 6000 to 1000, 1 KV head, 13.7 and 14.8; 1 x 16000 to 1000, 8 KV heads,
  // 25.2 (16) and 28.1 (32); 1 x 20000 30.6 (32) and 35.8 (passes).
  const int per = (p.max_ctx + kSelectThreads - 1) / kSelectThreads;
  if (items <= kSmallItems && per <= 32)
    return per <= 8    ? launch_small<8>(p, items, stream)
           : per <= 16 ? launch_small<16>(p, items, stream)
                       : launch_small<32>(p, items, stream);
  const hipError_t e = per <= 8    ? launch_select<8>(p, stream)
                       : per <= 16 ? launch_select<16>(p, stream)
                       : per <= 32 ? launch_select<32>(p, stream)
                                   : launch_select<0>(p, stream);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)std::min<int64_t>(items, kMaxMoveGrid)), block(kMoveThreads);
  // With a workgroup per compute unit or fewer, more blocks at a time save waits
  // (us a call with eight and four: 1 x 40000 to 4000, 1 KV head, 41.8 and 43.7; 1 x
  // 20000 to 1000, 8 of them, 36.1 and 38.0); with more of them, four leave room in
  // LDS for three on a unit (16 x 16K: the move 340 and 194).
  const bool few = items <= 256;
  if (p.src.vb_shift == 4)
    return few ? launch_kernel(evict_move_kernel<16, 8>, grid, block, stream, p)
               : launch_kernel(evict_move_kernel<16, 4>, grid, block, stream, p);
  return few ? launch_kernel(evict_move_kernel<32, 8>, grid, block, stream, p)
             : launch_kernel(evict_move_kernel<32, 4>, grid, block, stream, p);
}

}  // namespace hswa
