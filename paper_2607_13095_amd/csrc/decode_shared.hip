// Decode for batches in which runs of consecutive sequences share a prefix
// ("SWA-Aware Prefix Cache Tree": equal token prefixes share their cached
// slots): the prefix's keys are read once for all sequences of a run instead of
// once for each.
//
// Attention over a split key range is merged by the log-sum-exp identity, so a
// row is the merge of its part over the prefix and its part over the
// sequence's own keys. Two kernels:
//   work    one workgroup per compute unit, of one of two kinds:
//           prefix: all queries of a group against the shared keys, tiles of 64
//             keys in LDS under up to 256 columns, a column being a (sequence,
//             query, head) of one KV head. Bound by the matrix products and the
//             exponentials where the group is large, by reading the keys where
//             it is small.
//           own: the keys behind the prefix, one sequence at a time, a span of
//             32-key chunks per wave (decode_kernels.h). Bound by reading them.
//           The plan (plan_small) divides the compute units between the two by
//           what each has to do, so that matrix products and reads run side by
//           side. (As kernels one after the other, 32 sequences of 100 - 1500
//           own keys over 8192 shared ones took 23 + 26 us and their merge, all 38 so.)
//   merge   the partials of each row
// Every workgroup finds the plan by itself, in one wave: a kernel for it
// took 9 us. Batches of more than 64 sequences or 63 groups (or 2^31 own chunks)
// have that kernel (shared_plan_kernel).
// The key tiles of all (group, KV head, 256 columns), in that order, are cut into
// equal spans, one per prefix workgroup. Where there are few of these column
// tiles, each is padded to a multiple of a span, so that none crosses from one to
// the next (a second start took such a workgroup 8 of 37 us). Its two phases
// (matrix products, softmax with the staging of tiles) alternate between two
// groups of four waves, one wave of each on a SIMD, as in prefill.hip. Every
// shared tile is whole and seen by every query, so it needs no masks.
#include <algorithm>
#include <type_traits>

#include "decode_kernels.h"

namespace hswa {
namespace {

constexpr int kPlanThreads = 256;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kGroupLanes = 16;     // lanes that look over a group's sequences
constexpr int kThreads = 512;
constexpr int kKT = kSharedTile;    // keys per tile
constexpr int kBufs = 4;            // LDS tile buffers: two being read, one stored, one loading
constexpr int kTileCols = kSharedCols;  // columns of a workgroup
constexpr int kKTileBytes = kKT * kHeadDim * 2;
constexpr int kBufBytes = 2 * kKTileBytes;
constexpr int kStage = kKT * kHeadDim / 8 / kThreads;  // 16-byte pieces per thread per tile (K or V)
static_assert(kStage == 2, "piece i of a thread belongs to 32-key block i");
constexpr int kAhead = 4;           // LDS operand reads in flight ahead of the matrix products
constexpr float kLaneSumLimit = 4096.f;  // a lane's share of a row sum above which the running maximum is raised
constexpr int kMinSpan = 4;         // least key tiles of a span
constexpr int kMinOwn = 4;          // least chunks of a span of the own keys
constexpr int kXcds = 8;
constexpr int kWorkWaves = kThreads / kWave;
// What work takes, in 0.1 us (measured in place, with the other kind at work too; the
// slowest workgroups count): a key tile under up to 128 and under 256 columns; a
// workgroup's start and end on a span of them; a wave's chunk of own keys with the
// other seven at work (50 GB/s, what a compute unit gets from HBM whatever is in
// flight, would be 26) and its start; all compute units' share of a chunk at 5.5
// TB/s; the merge of a prefix workgroup's partials. (Against means, 10, 26 and 65
// for the first, the chunk and its start: 32 x (8192 + 100 - 1500) 40.9 us, now 38.4;
// 64 x (64K + 200 - 2000) 184, 178; 90 in 3 groups 60.8, 57.0.)
constexpr int kCostHalf = 14, kCostFull = 19;
constexpr float kCostSpan = 115.f;
constexpr float kCostOwn = 33.f, kCostOwnStart = 85.f, kCostOwnHbm = .03f, kCostMerge = .4f;
constexpr int kAlignedGroups = 16;  // up to this many groups the plan looks for spans that end with the tiles

__device__ __forceinline__ int64_t max64(int64_t a, int64_t b) { return a > b ? a : b; }
__device__ __forceinline__ int64_t ceil_div(int64_t a, int64_t b) {  // a >= 0, b > 0
  if (((a + b) >> 31) == 0) return ((uint32_t)a + (uint32_t)b - 1) / (uint32_t)b;  // (much shorter)
  return (a + b - 1) / b;
}
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {  // likewise
  return ((a | b) >> 31) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Inclusive scan over the workgroup of the plan with `op`; `last`: the result of all.
template <typename Op>
__device__ __forceinline__ int64_t block_scan(int64_t x, int64_t (&part)[kPlanWaves], int64_t &last, Op op) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  x = wave_scan(x, (int64_t)0, op);  // (sums and maxima of what is not negative)
  __syncthreads();  // (part was read by the scan before)
  if (lane == kWave - 1) part[wave] = x;
  __syncthreads();
  last = part[0];
#pragma unroll
  for (int w = 1; w < kPlanWaves; ++w) {
    if (w == wave) x = op(x, last);
    last = op(last, part[w]);
  }
  return x;
}

__device__ __forceinline__ int64_t cols_cost(int cols) {  // of a key tile under all columns of a group
  const int full = cols / kTileCols, rest = cols - full * kTileCols;
  return (int64_t)full * kCostFull + (rest == 0 ? 0 : rest <= kTileCols / 2 ? kCostHalf : kCostFull);
}

// The division of the compute units, by one wave: `units` key tiles that take
// `cost` in all, `chunks` chunks of own keys (of every KV head), at most `longest`
// of one sequence. Lane l tries 8 (l + 1) prefix workgroups.
__device__ __forceinline__ SharedHead divide_work(const DecodeParams &d, int64_t units, int64_t cost, int64_t chunks,
                                                  int64_t longest) {
  const int lane = threadIdx.x & (kWave - 1);
  int n = 0;
  if (units > 0) {
    const int mine = kXcds * (min(lane, kSharedSpans / kXcds - 1) + 1);
    const float u = (float)units, o = (float)chunks;
    const float per = fmaxf((float)kMinSpan, ceilf(u / mine));
    const float own_per = fmaxf((float)kMinOwn, ceilf(o / (max(kSharedSpans - mine, 1) * kWorkWaves)));
    const float own = o == 0.f ? 0.f : mine == kSharedSpans ? FLT_MAX : kCostOwnStart + fmaxf(own_per * kCostOwn, o * kCostOwnHbm);
    const float t = fmaxf(kCostSpan + per * ((float)cost / u), own) + mine * kCostMerge;
    const float least = last_lane(wave_scan(t, FLT_MAX, [](float a, float b) { return fminf(a, b); }));
    n = kXcds * (__builtin_ctzll(__ballot(t == least)) + 1);
  }
  SharedHead h;
  h.units = units;
  h.prefix_groups = n;
  h.per = n > 0 ? max64(kMinSpan, ceil_div(units, n)) : 1;
  // spans of the own keys: at most max_splits pieces of a sequence's
  const int waves = max(kSharedSpans - n, 1) * kWorkWaves;
  h.own.units = chunks;
  h.own.per = max64(max64(kMinOwn, ceil_div(chunks, waves)), ceil_div(longest, d.max_splits - 1));
  h.own.aligned = 0;
  return h;
}

// A plan's groups, by one wave that holds group l in lane l (tiles 0: none, or no
// group): the division of the compute units, the spans, the sums before each group.
__device__ __forceinline__ SharedHead plan_groups(const SharedParams &p, SharedGroup &g, int64_t chunks, int64_t longest,
                                                  int64_t &units_before, int64_t &rows_before) {
  const DecodeParams &d = p.d;
  const int lane = threadIdx.x & (kWave - 1);
  const auto add = [](auto a, auto b) { return a + b; };
  const int runs = d.hkv * ((g.cols + kTileCols - 1) / kTileCols);  // column tiles of all KV heads
  const int64_t rows = (int64_t)d.hkv * ((g.cols + kCols - 1) / kCols * kCols);
  rows_before = wave_scan(rows, (int64_t)0, add) - rows;
  const int64_t cost = wave_scan(d.hkv * cols_cost(g.cols) * g.tiles, (int64_t)0, add);
  int64_t u = (int64_t)runs * g.tiles, s = wave_scan(u, (int64_t)0, add);
  SharedHead h = divide_work(d, uni64(__shfl(s, kWave - 1, kWave)), uni64(__shfl(cost, kWave - 1, kWave)), chunks,
                             longest);
  g.padded = g.tiles;
  if (h.units > 0 && p.ng <= kAlignedGroups) {
    const int per = (int)min(h.per, (int64_t)INT32_MAX / 2) + lane;  // lane l tries this span
    int64_t spans = 0;
    for (int i = 0; i < p.ng; ++i) {
      const int t = __builtin_amdgcn_readlane(g.tiles, i);
      spans += (int64_t)__builtin_amdgcn_readlane(runs, i) * (int)((uint32_t)(t + per - 1) / (uint32_t)per);
    }
    const uint64_t fits = __ballot(spans <= h.prefix_groups);
    if (fits != 0) {
      h.per = __builtin_amdgcn_readlane(per, __builtin_ctzll(fits));
      const int at = (int)h.per;
      g.padded = (int)((uint32_t)(g.tiles + at - 1) / (uint32_t)at) * at;
      u = (int64_t)runs * g.padded;
      s = wave_scan(u, (int64_t)0, add);
      h.units = uni64(__shfl(s, kWave - 1, kWave));
    }
  }
  units_before = s - u;
  return h;
}

// The keys that a group shares, in tiles: every query of its sequences sees them
// (`least`: the shortest context, `count` sequences with one).
__device__ __forceinline__ int shared_tiles(const SharedParams &p, int shared, int least, int count) {
  const int n = min(min(shared, p.max_shared), min(least, p.d.max_ctx) - p.d.nq + 1);
  return count >= (p.cu_groups ? 2 : 1) && n > 0 ? n / kKT : 0;
}
// Group i's first sequence and the length that its sequences share, as given.
__device__ __forceinline__ int group_first(const SharedParams &p, int i) { return p.cu_groups ? p.cu_groups[i] : i; }
__device__ __forceinline__ int group_shared(const SharedParams &p, int i) {
  return p.cu_groups ? p.shared_lens[i] : INT32_MAX;
}

// The plan of a batch of up to 64 sequences and 63 groups, by one wave: lane l
// holds sequence l and group l. Every workgroup writes it to memory (the same
// values), where its waves on own keys and the merge read it, and what a prefix
// workgroup needs to LDS.
struct SmallPlan {
  SharedHead head;
  SharedGroup groups[kWave];
  int64_t units[kWave], rows[kWave];
  int least[kWave];
};
__device__ __forceinline__ void plan_small(const SharedParams &p, SmallPlan &at) {
  const DecodeParams &d = p.d;
  const int lane = threadIdx.x & (kWave - 1);
  const int ctx = lane < d.ns ? min(d.ctx_lens[lane], d.max_ctx) : 0;
  // offsets that are out of range or decrease make empty groups, never overlapping ones
  int cut = lane <= p.ng ? min(max(group_first(p, lane), 0), d.ns) : 0;
  const int shared = lane < p.ng ? group_shared(p, lane) : 0;
  cut = wave_scan(cut, 0, [](int a, int b) { return max(a, b); });
  const int end = __shfl(cut, min(lane + 1, kWave - 1), kWave);  // of group `lane` (lane < ng)
  const int all = __builtin_amdgcn_readlane(cut, p.ng);
  int grp = 0;  // of sequence `lane`: the last group that starts at or before it
  for (int i = 1; i < p.ng; ++i) grp = __builtin_amdgcn_readlane(cut, i) <= lane ? i : grp;
  const bool member = lane >= __builtin_amdgcn_readlane(cut, 0) && lane < all;
  grp = member ? grp : -1;
  // the shortest context of each group
  at.least[lane] = INT32_MAX;
  wave_exchange();
  if (member && ctx >= 1) atomicMin(&at.least[grp], ctx);
  wave_exchange();
  const uint64_t live = __ballot(ctx >= 1);
  const uint64_t upto = end >= 64 ? ~0ull : ((uint64_t)1 << end) - 1;
  const bool group = lane < p.ng && cut < end;
  const uint64_t mine = group ? live & upto & ~(((uint64_t)1 << cut) - 1) : 0;
  SharedGroup g;
  g.first = cut;
  g.leader = mine != 0 ? __builtin_ctzll(mine) : 0;
  g.tiles = group ? shared_tiles(p, shared, at.least[lane], __popcll(mine)) : 0;
  g.cols = g.tiles > 0 ? (end - cut) * d.nq * d.group : 0;
  const int tiles = __shfl(g.tiles, max(grp, 0), kWave);
  const int start = member && ctx >= 1 ? tiles * kKT : 0;
  const int nch = ctx >= 1 ? (ctx - start + kChunk - 1) / kChunk : 0;
  const int sc = wave_scan(nch, 0, [](int a, int b) { return a + b; });
  const int longest = __builtin_amdgcn_readlane(wave_scan(nch, 0, [](int a, int b) { return max(a, b); }), kWave - 1);
  const int H = d.hkv * ((d.nq * d.group + d.item_cols - 1) / d.item_cols);
  int64_t units, rows;
  SharedHead h = plan_groups(p, g, (int64_t)__builtin_amdgcn_readlane(sc, kWave - 1) * H, longest, units, rows);
  // Spans of the own keys that end with their sequence and KV head: a wave that
  // goes on with the next one starts anew there (3.5 us of about 20), which is
  // worth a chunk more a span (2.6 us), not two.
  int64_t before = (int64_t)(sc - nch) * H;
  {
    const int waves = (kSharedSpans - h.prefix_groups) * kWorkWaves / H;  // for each (KV head, column item)
    const int segments = __popcll(__ballot(nch > 0));
    if (waves > segments) {
      int per = (int)h.own.per;
      for (int tries = 0; tries < 2; ++tries, ++per) {
        const int mine = (int)((uint32_t)(nch + per - 1) / (uint32_t)per);
        const int all = wave_scan(mine, 0, [](int a, int b) { return a + b; });
        if (__builtin_amdgcn_readlane(all, kWave - 1) <= waves) {
          h.own = OwnSpans{(int64_t)__builtin_amdgcn_readlane(all, kWave - 1) * per * H, per, 1};
          before = (int64_t)(all - mine) * per * H;
          break;
        }
      }
    }
  }
  if (lane < p.ng) {
    p.groups[lane] = at.groups[lane] = g;
    p.group_units[lane] = at.units[lane] = units;
    p.group_rows[lane] = at.rows[lane] = rows;
  }
  // (the exchanges need every lane)
  SharedSeq q;
  const int from = max(grp, 0), first = __shfl(g.first, from, kWave);
  q.start = start;
  q.col = (lane - first) * d.nq * d.group;
  q.tiles = tiles;
  q.padded = __shfl(g.padded, from, kWave);
  q.cols = __shfl(g.cols, from, kWave);
  q.units = __shfl(units, from, kWave);
  q.rows = __shfl(rows, from, kWave);
  q.own_units = before;
  if (lane < d.ns) {
    p.start[lane] = start;
    p.own_units[lane] = before;
    p.seqs[lane] = q;
  }
  if (lane == 0) {
    p.group_units[p.ng] = at.units[p.ng] = h.units;
    *p.head = at.head = h;
  }
}

// The plan of a batch of up to kPlanThreads sequences and fewer groups, a thread
// each. (us a call with it and with the loops below: 90 sequences in 3 groups 60.8
// and 63.2, 256 in 100 groups 132.2 and 138.8, 64 / 8 heads; 200 in 30, 8 / 1, 43.1
// and 46.6.)
struct BlockPlan {
  int64_t part[kPlanWaves];
  int32_t cut[kPlanThreads];
  int32_t least[kPlanThreads], count[kPlanThreads], leader[kPlanThreads];
  SharedGroup groups[kPlanThreads];
  int64_t units[kPlanThreads], rows[kPlanThreads];
};
__device__ __forceinline__ void plan_block(const SharedParams &p, BlockPlan &at) {
  const DecodeParams &d = p.d;
  const int tid = threadIdx.x;
  const auto add = [](int64_t a, int64_t b) { return a + b; };
  const auto most = [](int64_t a, int64_t b) { return max64(a, b); };
  const int ctx = tid < d.ns ? min(d.ctx_lens[tid], d.max_ctx) : 0;
  const int shared = tid < p.ng ? group_shared(p, tid) : 0;
  // offsets that are out of range or decrease make empty groups, never overlapping ones
  const int cut = tid <= p.ng ? min(max(group_first(p, tid), 0), d.ns) : 0;
  int64_t last;
  at.cut[tid] = (int)block_scan(cut, at.part, last, most);
  at.least[tid] = at.leader[tid] = INT32_MAX;
  at.count[tid] = 0;
  __syncthreads();
  int grp = 0;  // of sequence `tid`: the last group that starts at or before it
  for (int hi = p.ng; hi - grp > 1;) {
    const int mid = (grp + hi) >> 1;
    if (at.cut[mid] <= tid) grp = mid;
    else hi = mid;
  }
  const bool member = tid >= at.cut[0] && tid < at.cut[p.ng] && ctx >= 1;
  if (member) {
    atomicMin(&at.least[grp], ctx);
    atomicMin(&at.leader[grp], tid);
    atomicAdd(&at.count[grp], 1);
  }
  __syncthreads();
  SharedGroup g{};
  if (tid < p.ng) {
    const int n = at.cut[tid + 1] - at.cut[tid];
    g.first = at.cut[tid];
    g.leader = at.count[tid] > 0 ? at.leader[tid] : 0;
    g.tiles = g.padded = n > 0 ? shared_tiles(p, shared, at.least[tid], at.count[tid]) : 0;
    g.cols = g.tiles > 0 ? n * d.nq * d.group : 0;
    at.groups[tid] = g;
  }
  __syncthreads();
  const int start = member ? at.groups[grp].tiles * kKT : 0;
  const int nch = ctx >= 1 ? (ctx - start + kChunk - 1) / kChunk : 0;
  const int H = d.hkv * ((d.nq * d.group + d.item_cols - 1) / d.item_cols);
  int64_t chunks, longest;
  const int64_t before = (block_scan(nch, at.part, chunks, add) - nch) * H;
  block_scan(nch, at.part, longest, most);
  int64_t units = 0, rows = 0, all_units = 0, cost = 0;
  if (p.ng >= kWave) {
    const int64_t gu = (int64_t)d.hkv * ((g.cols + kTileCols - 1) / kTileCols) * g.tiles;
    const int64_t gr = (int64_t)d.hkv * ((g.cols + kCols - 1) / kCols * kCols);
    units = block_scan(gu, at.part, all_units, add) - gu;
    rows = block_scan(gr, at.part, last, add) - gr;
    block_scan(d.hkv * cols_cost(g.cols) * g.tiles, at.part, cost, add);
  }
  if (tid < kWave) {
    const SharedHead h = p.ng < kWave ? plan_groups(p, g, chunks * H, longest, units, rows)
                                      : divide_work(d, all_units, cost, chunks * H, longest);
    if (tid == 0) {
      p.group_units[p.ng] = h.units;
      *p.head = h;
    }
  }
  if (tid < p.ng) {
    p.groups[tid] = at.groups[tid] = g;
    p.group_units[tid] = at.units[tid] = units;
    p.group_rows[tid] = at.rows[tid] = rows;
  }
  __syncthreads();
  if (tid >= d.ns) return;
  SharedSeq q{};
  q.start = start;
  q.own_units = before;
  if (start > 0) {
    g = at.groups[grp];
    q.col = (tid - g.first) * d.nq * d.group;
    q.tiles = g.tiles;
    q.padded = g.padded;
    q.cols = g.cols;
    q.units = at.units[grp];
    q.rows = at.rows[grp];
  }
  p.start[tid] = start;
  p.own_units[tid] = before;
  p.seqs[tid] = q;
}

__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(SharedParams p) {
  __shared__ BlockPlan plan;
  if (p.d.ns <= kPlanThreads && p.ng < kPlanThreads) {
    plan_block(p, plan);
    return;
  }
  auto &part = plan.part;
  __shared__ int32_t cut[kPlanThreads + 1];  // first sequences of the groups at hand, made non-decreasing
  const auto add = [](int64_t a, int64_t b) { return a + b; };
  const auto most = [](int64_t a, int64_t b) { return max64(a, b); };
  const DecodeParams &d = p.d;
  const int tid = threadIdx.x;
  for (int b = tid; b < d.ns; b += kPlanThreads) {
    p.start[b] = 0;
    p.group_of[b] = -1;
  }
  int64_t units = 0, rows = 0, cost = 0;  // before the groups at hand
  int carry = 0;
  for (int i0 = 0; i0 < p.ng; i0 += kPlanThreads) {
    const int n = min(kPlanThreads, p.ng - i0);
    // offsets that are out of range or decrease make empty groups, never overlapping ones
    auto offset = [&](int i) { return (int64_t)min(max(group_first(p, i0 + i), 0), d.ns); };
    int64_t all;
    const int64_t c = block_scan(max64(tid < n ? offset(tid) : 0, carry), part, all, most);
    if (tid < n) cut[tid] = (int)c;
    if (tid == 0) cut[n] = (int)max64(all, offset(n));
    __syncthreads();
    carry = cut[n];
    const int gl = tid & (kGroupLanes - 1);
    for (int i = tid / kGroupLanes; i < n; i += kPlanThreads / kGroupLanes) {
      const int first = cut[i], end = cut[i + 1];
      // its sequences with a context: the shortest context, their number, the first of them
      int least = d.max_ctx, count = 0, leader = end;
      for (int b = first + gl; b < end; b += kGroupLanes) {
        const int ctx = d.ctx_lens[b];
        if (ctx >= 1) {
          least = min(least, ctx);
          leader = min(leader, b);
          ++count;
        }
      }
#pragma unroll
      for (int off = 1; off < kGroupLanes; off <<= 1) {
        least = min(least, __shfl_xor(least, off, kGroupLanes));
        leader = min(leader, __shfl_xor(leader, off, kGroupLanes));
        count += __shfl_xor(count, off, kGroupLanes);
      }
      const int tiles = shared_tiles(p, group_shared(p, i0 + i), least, count);
      if (gl == 0) {
        SharedGroup g;
        g.first = first;
        g.leader = leader;
        g.tiles = g.padded = tiles;
        g.cols = tiles > 0 ? (end - first) * d.nq * d.group : 0;
        p.groups[i0 + i] = g;
      }
      if (tiles > 0)
        for (int b = first + gl; b < end; b += kGroupLanes) {
          p.start[b] = d.ctx_lens[b] >= 1 ? tiles * kKT : 0;
          p.group_of[b] = i0 + i;
        }
    }
    __syncthreads();
    int64_t gu = 0, gr = 0, gc = 0;
    if (tid < n) {
      const SharedGroup &g = p.groups[i0 + tid];
      gu = (int64_t)d.hkv * ((g.cols + kTileCols - 1) / kTileCols) * g.tiles;
      gr = (int64_t)d.hkv * ((g.cols + kCols - 1) / kCols * kCols);
      gc = d.hkv * cols_cost(g.cols) * g.tiles;
    }
    int64_t tu, tr, tc;
    const int64_t su = block_scan(gu, part, tu, add), sr = block_scan(gr, part, tr, add);
    block_scan(gc, part, tc, add);
    if (tid < n) {
      p.group_units[i0 + tid] = units + su - gu;
      p.group_rows[i0 + tid] = rows + sr - gr;
    }
    units += tu;
    rows += tr;
    cost += tc;
  }
  // the own keys, in chunks
  __syncthreads();
  const int H = d.hkv * ((d.nq * d.group + d.item_cols - 1) / d.item_cols);
  int64_t chunks = 0, longest = 0;
  for (int b0 = 0; b0 < d.ns; b0 += kPlanThreads) {
    const int64_t n = seq_chunks<kSuffix>(d, b0 + tid);
    int64_t total, m;
    const int64_t s = block_scan(n, part, total, add);
    block_scan(n, part, m, most);
    if (b0 + tid < d.ns) p.own_units[b0 + tid] = (chunks + s - n) * H;
    chunks += total;
    longest = max64(longest, m);
  }
  if (tid < kWave) {
    SharedHead h;
    if (p.ng < kWave) {  // few groups: as in a small plan
      SharedGroup g{};
      if (tid < p.ng) g = p.groups[tid];
      int64_t before, first;
      h = plan_groups(p, g, chunks * H, longest, before, first);
      if (tid < p.ng) {
        p.groups[tid] = g;
        p.group_units[tid] = before;
        p.group_rows[tid] = first;
      }
    } else {
      h = divide_work(d, units, cost, chunks * H, longest);
    }
    if (tid == 0) {
      p.group_units[p.ng] = h.units;
      *p.head = h;
    }
  }
  __syncthreads();
  for (int b = tid; b < d.ns; b += kPlanThreads) {
    SharedSeq q{};
    q.start = p.start[b];
    q.own_units = p.own_units[b];
    if (q.start > 0) {
      const int i = p.group_of[b];
      const SharedGroup g = p.groups[i];
      q.col = (b - g.first) * d.nq * d.group;
      q.tiles = g.tiles;
      q.padded = g.padded;
      q.cols = g.cols;
      q.units = p.group_units[i];
      q.rows = p.group_rows[i];
    }
    p.seqs[b] = q;
  }
}

struct __attribute__((aligned(16))) TileBufs {
  unsigned char b[kBufs * kBufBytes];
};

// Key tiles [j0, j1) of a group (its leader's row of the block table) for KV
// head g and the columns from col0 on: partial rows to slot, slot + 1, ... of
// the workspace. kCG: 16-column groups of a wave. kPage: keys of a page, 64
// standing for 64 and more. kMode: as for the own keys.
template <int kCG, int kPage, int kMode>
__device__ __forceinline__ void prefix_tiles(const SharedParams &p, TileBufs &bufs, const SharedGroup &grp, int g,
                                             int col0, int j0, int j1, int64_t slot) {
  unsigned char *const s_lds = bufs.b;
  const DecodeParams &d = p.d;
  const PoolView &pv = d.pool;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int r = lane & 15, q = lane >> 4;
  const int shift = pv.pg_shift;
  const float c2 = d.scale_log2;
  const int ncols = min(grp.cols - col0, kTileCols);
  // column group cg of the wave: columns 16 (8 cg + wave) .. + 15
  const bool active = 16 * wave < ncols;  // (the first one; a wave without columns only stages)

  // ---- staging: global -> registers -> LDS, in MFMA operand order ----
  // K: the pool's 32-key blocks as they are; V^T: block (h, dt) holds, for lane
  // r + 16 q, keys 32 h + 8 q .. + 7 of dim 16 dt + r.
  constexpr int kPages = kKT / kPage;
  const int vq = (tid >> 4) & 3, vdim = 16 * (tid >> 6) + (tid & 15);
  const int last_lp = (kKT * j1 - 1) >> shift;
  int tab_lp0 = (kKT * j0) >> shift;
  auto load_tab = [&](int lp0) {  // lane i: the entry of logical page lp0 + i
    const int lp = lp0 + lane;
    return lp <= last_lp ? pv.table[(int64_t)grp.leader * pv.stride + lp] : -1;
  };
  int tab_page = load_tab(tab_lp0), tab_next = load_tab(tab_lp0 + kWave);
  u32x4 qf[kCG][4];
#pragma unroll
  for (int cg = 0; cg < kCG; ++cg) {
    const int col = 16 * (8 * cg + wave) + r;
    const bool valid = col < ncols;
    const int x = col0 + (valid ? col : 0), per = d.nq * d.group;
    const int m = x / per, rem = x - m * per, qi = rem / d.group, hh = rem - qi * d.group;
    const uint16_t *qrow =
        d.q + (((int64_t)(grp.first + m) * d.nq + qi) * d.hq + (int64_t)g * d.group + hh) * kHeadDim;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const u32x4 v = ldg128(qrow + 32 * t + 8 * q);
      const u32x4 z = {0u, 0u, 0u, 0u};
      qf[cg][t] = valid ? v : z;
    }
  }

  // this thread's pieces of a tile (opaque, so that the second's stays an offset of its own)
  uint32_t koff[kStage], voff[kStage];
#pragma unroll
  for (int i = 0; i < kStage; ++i) {
    const uint32_t blk = kPage == 64 ? 8192u * i : 0u;
    koff[i] = kPage == 16 ? (uint32_t)((tid >> 4) * 128 + (tid & 7) * 16) : blk + (uint32_t)tid * 16u;
    voff[i] = kPage == 16 ? (uint32_t)(vdim * 32 + (vq & 1) * 16) : blk + (uint32_t)(vdim * 32 + vq * 8) * 2u;
    asm volatile("" : "+v"(koff[i]), "+v"(voff[i]));
  }
  uint32_t held = 0;  // bit 4 (j % 8) + n: the n-th 16 keys of tile j are in the pool
  u32x4 sk[kStage], sv[kStage];
  auto fetch = [&](int j, u32x4 (&k)[kStage], u32x4 (&v)[kStage]) __attribute__((always_inline)) {
    const int kt = kKT * j, lp = kt >> shift;
    if (lp - tab_lp0 >= kWave) {
      tab_lp0 += kWave;
      tab_page = tab_next;
      tab_next = load_tab(tab_lp0 + kWave);
    }
    int page[kPages];
    uint32_t bits = 0;
#pragma unroll
    for (int n = 0; n < kPages; ++n) {
      const int e = __builtin_amdgcn_readlane(tab_page, lp + n - tab_lp0);
      page[n] = e >= 0 && e < pv.num_pages ? e : -1;
      bits |= page[n] >= 0 ? ((1u << (4 / kPages)) - 1u) << (n * (4 / kPages)) : 0u;
    }
    const int at = 4 * (j & 7);
    held = (held & ~(15u << at)) | (bits << at);
    auto page_off = [&](int pg) {  // byte offset of the page-head (of the tile in it)
      const uint64_t o = ((uint64_t)((uint32_t)max(pg, 0)) * (uint32_t)d.hkv + (uint32_t)g) << (shift + kHeadDimShift + 1);
      return kPage == 64 ? o + ((uint64_t)((uint32_t)kt & ((1u << shift) - 1u)) << (kHeadDimShift + 1)) : o;
    };
    // Bases are wave-uniform, a lane adds a fixed offset: buffer loads, without
    // vector address arithmetic (with 16-key pages a lane chooses one of two).
    auto load = [&](const uint16_t *pool, uint64_t o, uint32_t lane_off) __attribute__((always_inline)) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char *>(reinterpret_cast<const char *>(pool)) + o, 0, kKTileBytes, kBufferWord3);
      return __builtin_amdgcn_raw_buffer_load_b128(rs, (int)lane_off, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kStage; ++i) {
      if constexpr (kPage == 16) {
        const uint64_t o0 = page_off(page[2 * i]), o1 = page_off(page[2 * i + 1]);
        const uint64_t ko = tid & 8 ? o1 : o0, vo = vq & 2 ? o1 : o0;  // of this lane's K rows and V keys
        k[i] = ldg128_global(reinterpret_cast<const char *>(pv.k_pool) + ko + koff[0]);
        v[i] = ldg128_global(reinterpret_cast<const char *>(pv.v_pool) + vo + voff[0]);
      } else {
        const uint64_t o = page_off(page[kPage == 32 ? i : 0]);
        k[i] = load(pv.k_pool, o, koff[i]);
        v[i] = load(pv.v_pool, o, voff[i]);
      }
    }
    if (bits != 15u) {  // a page outside the pool: its keys are left out, their values zero
#pragma unroll
      for (int i = 0; i < kStage; ++i) {
        const u32x4 z = {0u, 0u, 0u, 0u};
        v[i] = (bits >> (2 * i + (vq >> 1))) & 1u ? v[i] : z;
      }
    }
  };
  auto buf_off = [&](int buf) { return (uint32_t)__builtin_amdgcn_readfirstlane(buf * kBufBytes); };
  auto lds128 = [&](uint32_t off) { return reinterpret_cast<u32x4 *>(s_lds + off); };
  auto store_tile = [&](int buf, const u32x4 (&k)[kStage], const u32x4 (&v)[kStage]) __attribute__((always_inline)) {
    const uint32_t a = buf_off(buf) + tid * 16;
#pragma unroll
    for (int i = 0; i < kStage; ++i) {
      *lds128(a + i * (kKTileBytes / 2)) = k[i];
      *lds128(a + kKTileBytes + i * (kKTileBytes / 2)) = v[i];
    }
  };

  float m[kCG], lsum[kCG];
  f32x4 acc[kCG][8];
#pragma unroll
  for (int cg = 0; cg < kCG; ++cg) {
    m[cg] = -FLT_MAX;
    lsum[cg] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[cg][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const uint32_t op_lane = lane * 16;
  auto qk_half = [&](int buf, int h, f32x4 (&sc)[2][kCG]) {
    const uint32_t a = buf_off(buf) + op_lane + h * (kKTileBytes / 2);
#pragma unroll
    for (int cg = 0; cg < kCG; ++cg) sc[0][cg] = sc[1][cg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const u32x4 ka = *lds128(a + 1024 * t);
      const u32x4 kb = *lds128(a + 4096 + 1024 * t);
#pragma unroll
      for (int cg = 0; cg < kCG; ++cg) {
        sc[0][cg] = mfma16x16x32(ka, qf[cg][t], sc[0][cg]);
        sc[1][cg] = mfma16x16x32(kb, qf[cg][t], sc[1][cg]);
      }
    }
  };
  auto pv_tile = [&](int buf, const u32x4 (&pf)[2][kCG]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t a = buf_off(buf) + kKTileBytes + op_lane + h * (kKTileBytes / 2);
      u32x4 vf[8];
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) vf[dt] = *lds128(a + 1024 * dt);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt)
#pragma unroll
        for (int cg = 0; cg < kCG; ++cg) acc[cg][dt] = mfma16x16x32(vf[dt], pf[h][cg], acc[cg][dt]);
    }
  };
  // Exponentials against the running maximum as it stands; it is raised, and the
  // tile's exponentials taken again, only if some lane's share of a row sum
  // exceeds 2^12 (an infinite one counts): numerator and denominator share the
  // maximum, so the result is the same. It starts at -FLT_MAX, so that a masked
  // score gives 0 and the first finite one raises it. The probabilities go to the
  // PV product in bf16, as those of the own keys do (decode_kernels.h: why, and what
  // it costs); sums, maxima and partial rows are fp32.
  auto tile_exp = [&](const f32x4 (&sc)[2][2][kCG], u32x4 (&pf)[2][kCG], float (&ts)[kCG]) {
#pragma unroll
    for (int cg = 0; cg < kCG; ++cg) {
      const float mc = m[cg];
      ts[cg] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float pr[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) pr[e] = fast_exp2(fmaf(sc[h][e >> 2][cg][e & 3], c2, -mc));
#pragma unroll
        for (int j = 0; j < 4; ++j) pf[h][cg][j] = pack_bf16x2(pr[2 * j], pr[2 * j + 1]);
        if constexpr (scored(kMode)) {
          ts[cg] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) ts[cg] = dot2_bf16_ones(pf[h][cg][j], ts[cg]);
        }
      }
    }
  };
  auto softmax_tile = [&](int j, f32x4 (&sc)[2][2][kCG], u32x4 (&pf)[2][kCG]) {
    const uint32_t bits = (held >> (4 * (j & 7))) & 15u;
    if (bits != 15u) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool in = (bits >> (2 * h + (q >> 1))) & 1u;
#pragma unroll
        for (int cg = 0; cg < kCG; ++cg)
#pragma unroll
          for (int e = 0; e < 8; ++e) sc[h][e >> 2][cg][e & 3] = in ? sc[h][e >> 2][cg][e & 3] : -INFINITY;
      }
    }
    float ts[kCG];
    tile_exp(sc, pf, ts);
    bool raise = false;
#pragma unroll
    for (int cg = 0; cg < kCG; ++cg) raise = raise || !(ts[cg] <= kLaneSumLimit);
    if (__builtin_amdgcn_ballot_w64(raise) != 0) {
#pragma unroll
      for (int cg = 0; cg < kCG; ++cg) {
        float s8[2][8];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 8; ++e) s8[h][e] = sc[h][e >> 2][cg][e & 3];
        const float cmax = max_xor32(max_xor16(max2(max8(s8[0]), max8(s8[1])))) * c2;
        const bool up = cmax > m[cg];
        const float alpha = up ? fast_exp2(m[cg] - cmax) : 1.f;
        m[cg] = up ? cmax : m[cg];
        lsum[cg] *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[cg][dt] *= alpha;
      }
      tile_exp(sc, pf, ts);
    }
#pragma unroll
    for (int cg = 0; cg < kCG; ++cg) lsum[cg] += ts[cg];
  };

  const int ntiles = j1 - j0;
  {
    u32x4 k0[kStage], v0[kStage], k1[kStage], v1[kStage];
    fetch(j0, k0, v0);
    if (ntiles > 1) fetch(j0 + 1, k1, v1);
    if (ntiles > 2) fetch(j0 + 2, sk, sv);
    store_tile(0, k0, v0);
    if (ntiles > 1) store_tile(1, k1, v1);
  }
  __syncthreads();
  f32x4 sc[2][2][kCG];
  u32x4 pf[2][kCG];
  // matrix phase of tile jt (from j0 on): PV of tile jt - 1, QK^T of tile jt,
  // at raised issue priority, operand reads kAhead reads ahead of the products
  auto matrix_phase = [&](int jt, auto first_tag) __attribute__((always_inline)) {
    constexpr bool kFirst = decltype(first_tag)::value;
    constexpr int kReads = kFirst ? 16 : 32;
    if (!active) return;
    const int buf = jt & (kBufs - 1);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(2);
    if constexpr (!kFirst) pv_tile((jt + kBufs - 1) & (kBufs - 1), pf);
    qk_half(buf, 0, sc[0]);
    qk_half(buf, 1, sc[1]);
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int i = 0; i < kReads - kAhead; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kCG, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kCG * kAhead, 0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  };
  auto softmax_phase = [&](int jt) __attribute__((always_inline)) {
    if (jt + 2 < ntiles) store_tile((jt + 2) & (kBufs - 1), sk, sv);
    if (jt + 3 < ntiles) fetch(j0 + jt + 3, sk, sv);
    if (active) softmax_tile(j0 + jt, sc, pf);
  };
  auto tile_barrier = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
  };
  // One barrier per tile. Between barriers t and t + 1 waves 0-3 run the matrix
  // phase of tile t, then its softmax phase; waves 4-7 first the softmax phase
  // of tile t - 1, then the matrix phase of tile t. Read in between are tiles t
  // (K) and t - 1 (V), stored are tiles t + 2 (waves 0-3) and t + 1 (waves 4-7),
  // whose buffers were last read before barrier t.
  constexpr std::true_type kFirstTile{};
  constexpr std::false_type kNextTile{};
  if (wave < kThreads / kWave / 2) {
    matrix_phase(0, kFirstTile);
    softmax_phase(0);
    tile_barrier();
    for (int jt = 1; jt < ntiles; ++jt) {
      matrix_phase(jt, kNextTile);
      softmax_phase(jt);
      tile_barrier();
    }
  } else {
    matrix_phase(0, kFirstTile);
    tile_barrier();
    for (int jt = 1; jt < ntiles; ++jt) {
      softmax_phase(jt - 1);
      matrix_phase(jt, kNextTile);
      tile_barrier();
    }
    softmax_phase(ntiles - 1);
  }
  if (!active) return;
  pv_tile((ntiles + kBufs - 1) & (kBufs - 1), pf);
#pragma unroll
  for (int cg = 0; cg < kCG; ++cg) {
    const float l = sum_xor32(sum_xor16(lsum[cg]));
    const int col = 16 * (8 * cg + wave) + r;
    if (col >= ncols) continue;
    const float inv = l > 0.f ? 1.f / l : 0.f;  // (no key in the pool: o = 0, log-sum-exp -inf)
    float *dst = p.ws_o + (slot + col) * kHeadDim + 4 * q;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4 *>(dst + 16 * dt) = acc[cg][dt] * inv;
    if (q == 0) p.ws_lse[slot + col] = m[cg] + __log2f(l);
  }
}

// kCGd: 16-column groups of a wave of the own keys. kMode: kSuffix, kSuffixScored.
template <int kPage, int kCGd, int kMode>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void shared_work_kernel(SharedParams p) {
  __shared__ TileBufs bufs;
  __shared__ SmallPlan plan;
  const int wave = uni((int)(threadIdx.x / kWave));
  if (p.small) {
    if (wave == 0) plan_small(p, plan);
    __syncthreads();
  }
  const SharedHead head = p.small ? plan.head : *p.head;
  // Workgroup ids go to the XCDs round-robin. An XCD gets as many of each kind
  // as the others, and of the spans of key tiles consecutive ones, which read
  // the same keys for other columns, or neighbouring ones.
  const int xcd = (int)(blockIdx.x % kXcds), local = (int)(blockIdx.x / kXcds);
  const int each = uni(head.prefix_groups) / kXcds;
  if (local >= each) {
    const int64_t first = (int64_t)xcd * (kSharedSpans / kXcds - each) + (local - each);
    decode_waves<true, (kPage > 16), kCGd, kMode>(p.d, first * kWorkWaves + wave);
    return;
  }
  const int span = xcd * each + local;
  const int64_t per = uni64(head.per), units = uni64(head.units);
  int64_t u = span * per;
  const int64_t u1 = u + per < units ? u + per : units;
  if (u >= u1) return;
  auto units_before = [&](int i) { return uni64(p.small ? plan.units[i] : p.group_units[i]); };
  int gi = 0;  // the group holding unit u: the last one that starts at or before it
  for (int hi = p.ng; hi - gi > 1;) {
    const int mid = (gi + hi) >> 1;
    if (units_before(mid) <= u) gi = mid;
    else hi = mid;
  }
  for (;;) {
    while (u >= units_before(gi + 1)) ++gi;
    SharedGroup grp = p.small ? plan.groups[gi] : p.groups[gi];
    grp = SharedGroup{uni(grp.first), uni(grp.leader), uni(grp.tiles), uni(grp.padded), uni(grp.cols)};
    const int ntc = (grp.cols + kTileCols - 1) / kTileCols;
    const int64_t rem = u - units_before(gi);
    const int seg = (int)(rem / grp.padded), j0 = (int)(rem - (int64_t)seg * grp.padded);
    const int g = seg / ntc, col0 = (seg - g * ntc) * kTileCols;
    const int left = (int)min((int64_t)(grp.padded - j0), u1 - u);  // units of this column tile in the span
    const int j1 = min(grp.tiles, j0 + left);
    const int64_t rows = (grp.cols + kCols - 1) / kCols * kCols;
    // pieces follow each other by tile or by span: no two share a row
    const int64_t slot = uni64(p.small ? plan.rows[gi] : p.group_rows[gi]) + g * rows + col0 + (int64_t)span * kTileCols;
    if (j0 < j1) {
      if (grp.cols - col0 <= kTileCols / 2) prefix_tiles<1, kPage, kMode>(p, bufs, grp, g, col0, j0, j1, slot);
      else prefix_tiles<2, kPage, kMode>(p, bufs, grp, g, col0, j0, j1, slot);
    }
    u += left;
    if (u >= u1) return;
    __syncthreads();  // every wave has read the tile buffers
  }
}

// Merge of a row's pieces, those of the prefix and then its own: kRowWaves waves
// per row (see kWideMergeRows), each taking every kRowWaves-th 16 pieces; the two
// half-waves take even and odd ones, four output dims a lane. kSuffixScored: also
// writes the row's log-sum-exp (+infinity for a row that sees no key).
template <int kRowWaves, int kMode>
__global__ __launch_bounds__(kMergeThreads) void shared_merge_kernel(SharedParams p) {
  const DecodeParams &d = p.d;
  const int lane = threadIdx.x & (kWave - 1);
  constexpr int kMergeWaves = kMergeThreads / kWave;
  static_assert(kRowWaves == 1 || kRowWaves == kMergeWaves, "a row has one wave or its workgroup");
  const int wid = uni((int)(threadIdx.x / kWave));
  const int rw = kRowWaves == 1 ? 0 : wid;  // wave of the row
  const uint32_t idx = blockIdx.x * (kMergeWaves / kRowWaves) + (kRowWaves == 1 ? wid : 0);  // (below 2^26)
  const uint32_t each = d.nq * d.hq;
  if (idx >= d.ns * each) return;
  const int b = (int)(idx / each);
  // (the loads of all go out together)
  const int given = d.ctx_lens[b];
  const SharedHead h = *p.head;
  const SharedSeq seq = p.seqs[b];
  const int half = lane >> 5, d4 = (lane & 31) * 4;
  u32x2 *dst = reinterpret_cast<u32x2 *>(d.out + (int64_t)idx * kHeadDim + d4);
  const u32x2 zero = {0u, 0u};
  const int rem = (int)(idx - b * each);
  const int qi = (int)((uint32_t)rem / (uint32_t)d.hq), head = rem - qi * d.hq;
  const int g = (int)((uint32_t)head / (uint32_t)d.group), hh = head - g * d.group;
  const int ctx = min(given, d.max_ctx);
  if (ctx < 1) {
    if (half == 0) *dst = zero;
    if (scored(kMode) && lane == 0) d.row_lse[idx] = INFINITY;
    return;
  }
  // pieces of the prefix: rows first, first + 256, ... of its partials
  int n0 = 0;
  int64_t first = 0;
  if (seq.start > 0) {
    const int col = seq.col + qi * d.group + hh;
    const int ntc = (seq.cols + kTileCols - 1) / kTileCols;
    const int64_t u = seq.units + (int64_t)(g * ntc + col / kTileCols) * seq.padded;
    const int64_t s0 = quotient(u, h.per);
    n0 = (int)(quotient(u + seq.tiles - 1, h.per) - s0) + 1;
    first = seq.rows + (int64_t)g * ((seq.cols + kCols - 1) / kCols * kCols) + col + s0 * kTileCols;
  }
  // and of its own keys
  const int nch = (ctx - seq.start + kChunk - 1) / kChunk;
  int n1 = 0;
  if (nch > 0) {
    if (h.own.aligned) {
      n1 = (int)ceil_div(nch, h.own.per);
    } else {
      const int hchunks = (d.nq * d.group + d.item_cols - 1) / d.item_cols;
      const int64_t u = seq.own_units + (int64_t)(g * hchunks + (qi * d.group + hh) / d.item_cols) * nch;
      n1 = (int)(quotient(u + nch - 1, h.own.per) - quotient(u, h.own.per)) + 1;
    }
  }
  if (!scored(kMode) && n0 == 0 && n1 == 1) return;  // one piece: the decode kernel wrote the row
  const int n = n0 + n1;
  const float *po0 = p.ws_o + first * kHeadDim + d4, *po1 = d.ws_o + (int64_t)idx * d.max_splits * kHeadDim + d4;
  auto load = [&](int s0, f32x4 (&v)[8]) {  // pieces s0 .. s0 + 15
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = s0 + 2 * k + half;
      const f32x4 z = {0.f, 0.f, 0.f, 0.f};
      const float *src = s < n0 ? po0 + (int64_t)s * kTileCols * kHeadDim : po1 + (int64_t)(s - n0) * kHeadDim;
      v[k] = s < n ? *reinterpret_cast<const f32x4 *>(src) : z;
    }
  };
  f32x4 v[8];
  load(16 * rw, v);  // (beside the log-sum-exps)
  auto lse_of = [&](int s) {
    return s < n0 ? p.ws_lse[first + (int64_t)s * kTileCols] : d.ws_lse[(int64_t)idx * d.max_splits + s - n0];
  };
  float mx = -INFINITY;
  for (int s = lane; s < n; s += kWave) mx = fmaxf(mx, lse_of(s));
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, kWave));
  mx = max_xor32(max_xor16(mx));
  if (mx == -INFINITY) {  // a row that sees no key
    if (half == 0) *dst = zero;
    if (scored(kMode) && lane == 0) d.row_lse[idx] = INFINITY;
    return;
  }
  float wsum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < n; s0 += kWave) {
    const int s = s0 + lane;
    const float w = s < n ? fast_exp2(lse_of(s) - mx) : 0.f;
    const int m = min(kWave, n - s0);
    for (int k0 = 16 * rw; k0 < m; k0 += 16 * kRowWaves) {
      if (s0 + k0 != 16 * rw) load(s0 + k0, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float we = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k0 + 2 * k));
        const float wd = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k0 + 2 * k + 1));
        const float wk = half ? wd : we;  // (0 past the last piece)
        wsum += wk;
        o += wk * v[k];
      }
    }
  }
  wsum = sum_xor32(wsum);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = sum_xor32(o[i]);
  if constexpr (kRowWaves > 1) {
    __shared__ f32x4 s_o[kRowWaves][kWave / 2];
    __shared__ float s_w[kRowWaves];
    if (half == 0) s_o[rw][lane] = o;
    if (lane == 0) s_w[rw] = wsum;
    __syncthreads();
    if (rw != 0) return;
    wsum = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
      wsum += s_w[w];
      o += s_o[w][lane & 31];
    }
  }
  if (scored(kMode) && lane == 0) d.row_lse[idx] = mx + __log2f(wsum);
  const float inv = 1.f / wsum;
  if (half == 0) {
    u32x2 w2;
    w2[0] = pack_bf16x2(o[0] * inv, o[1] * inv);
    w2[1] = pack_bf16x2(o[2] * inv, o[3] * inv);
    *dst = w2;
  }
}

template <int kCGd, int kMode>
hipError_t launch_work(const SharedParams &p, hipStream_t stream) {
  const dim3 grid(kSharedSpans), threads(kThreads);
  switch (p.d.pool.pg_shift) {
    case 4: return launch_kernel(shared_work_kernel<16, kCGd, kMode>, grid, threads, stream, p);
    case 5: return launch_kernel(shared_work_kernel<32, kCGd, kMode>, grid, threads, stream, p);
    default: return launch_kernel(shared_work_kernel<64, kCGd, kMode>, grid, threads, stream, p);
  }
}

template <int kCGd, int kMode>
hipError_t launch_cg(const SharedParams &p0, hipStream_t stream) {
  SharedParams p = p0;
  DecodeParams &d = p.d;
  d.item_cols = kCGd * kCols;
  const int64_t chunks = (int64_t)d.ns * ((d.max_ctx + kChunk - 1) / kChunk);
  const int heads = d.hkv * ((d.nq * d.group + d.item_cols - 1) / d.item_cols);
  p.small = d.ns <= kWave && p.ng < kWave && chunks * heads <= INT32_MAX;  // (its sums are 32-bit)
  hipError_t e = p.small ? hipSuccess : launch_kernel(shared_plan_kernel, dim3(1), dim3(kPlanThreads), stream, p);
  if (e != hipSuccess) return e;
  if ((e = launch_work<kCGd, kMode>(p, stream)) != hipSuccess) return e;
  const int64_t rows = (int64_t)d.ns * d.nq * d.hq;
  constexpr int per_block = kMergeThreads / kWave;
  if (rows <= kWideMergeRows)
    return launch_kernel(shared_merge_kernel<per_block, kMode>, dim3((unsigned)rows), dim3(kMergeThreads), stream, p);
  return launch_kernel(shared_merge_kernel<1, kMode>, dim3((unsigned)((rows + per_block - 1) / per_block)),
                       dim3(kMergeThreads), stream, p);
}

}  // namespace

hipError_t launch_decode_shared(const SharedParams &p, hipStream_t stream) {
  return p.d.nq * p.d.group > kCols ? launch_cg<2, kSuffix>(p, stream) : launch_cg<1, kSuffix>(p, stream);
}

hipError_t launch_decode_shared_scored(const SharedParams &p, hipStream_t stream) {
  return launch_cg<2, kSuffixScored>(p, stream);  // (more than kKeepColumns columns)
}

}  // namespace hswa
