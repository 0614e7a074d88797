// Decode calls over the paged KV cache: span lengths, grids and launches (the
// kernels are in decode_kernels.h).
#include "decode_kernels.h"

namespace hswa {

int32_t decode_split_len(int32_t ns, int32_t hkv, int32_t group, int32_t max_ctx) {
  // The fewest keys of a wave's span: 256 to 2048, larger for larger batches
  // (about 8192 spans of this length when contexts average half the maximum),
  // so that spans of small batches stay short enough to fill the device and
  // the workspace stays bounded; very long contexts get longer spans so that a
  // row has at most 257 pieces.
  const int64_t heads = (int64_t)hkv * ((group + kCols - 1) / kCols);
  const int64_t keys = heads * ns * (int64_t)max_ctx / 2;
  int32_t len = 256;
  while (len < 2048 && keys / (2 * len) >= 8192) len *= 2;
  const int64_t min_len = ((int64_t)max_ctx + 255) / 256;
  while (len < min_len) len *= 2;
  return len;
}

template <int kCGd>
hipError_t launch_decode_cg(const DecodeParams &p0, hipStream_t stream) {
  DecodeParams p = p0;
  p.item_cols = kCols * kCGd;
  const int hitems = (p.nq * p.group + p.item_cols - 1) / p.item_cols;
  const int64_t items = (int64_t)p.ns * p.hkv * hitems;  // whole range: one item per workgroup
  // One-page path: 32-key chunks never straddle pages (PG >= 32).
  const bool one_page = p.pool.pg_shift >= 5;
  const dim3 block(kWave * kWaves);
  if (p.max_splits > 1) {
    hipError_t e = one_page ? resident_split_waves<true, kCGd>(p.span_waves)
                            : resident_split_waves<false, kCGd>(p.span_waves);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)(p.span_waves / kWaves));
    e = one_page ? launch_kernel(decode_kernel<true, true, kCGd>, grid, block, stream, p)
                 : launch_kernel(decode_kernel<true, false, kCGd>, grid, block, stream, p);
    if (e != hipSuccess) return e;
    const int64_t rows = (int64_t)p.ns * p.nq * p.hq;
    constexpr int per_block = kMergeThreads / kWave;
    if (rows <= kWideMergeRows)
      return launch_kernel(decode_merge_kernel<per_block>, dim3((unsigned)rows), dim3(kMergeThreads), stream, p);
    return launch_kernel(decode_merge_kernel<1>, dim3((unsigned)((rows + per_block - 1) / per_block)),
                         dim3(kMergeThreads), stream, p);
  }
  return one_page ? launch_kernel(decode_kernel<false, true, kCGd>, dim3((unsigned)items), block, stream, p)
                  : launch_kernel(decode_kernel<false, false, kCGd>, dim3((unsigned)items), block, stream, p);
}

hipError_t launch_decode(const DecodeParams &p, hipStream_t stream) {
  if (p.ns <= 0) return hipSuccess;
  // more than 16 (query, head) columns per KV head: one wave takes 32 of them
  return p.nq * p.group > kCols ? launch_decode_cg<2>(p, stream) : launch_decode_cg<1>(p, stream);
}

}  // namespace hswa
