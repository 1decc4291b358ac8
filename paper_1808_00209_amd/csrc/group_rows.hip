// Rows in the order of their group (bnn_group_rows): a stable counting sort
// in one launch.  Block g belongs to group g, block G to the rows of no
// group.  Every block reads all ids: once for the number of rows of lower
// groups, where its own begin, and once to write its own.  A wave takes a
// contiguous part of the ids, so that the order within a group is that of the
// rows and does not hang on any timing.
#include "experts.hpp"

namespace bnn {
namespace {

constexpr int kNT = 1024;
constexpr int kNW = kNT / 64;

__global__ __launch_bounds__(kNT) void group_rows_kernel(const int32_t* __restrict__ ids,
                                                         int32_t M, int32_t G,
                                                         int32_t* __restrict__ offsets,
                                                         int32_t* __restrict__ order) {
  __shared__ int32_t below[kNW], mine[kNW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = blockIdx.x;
  // (an id outside [0, G) counts as G)
  auto group_of = [&](int32_t id) {
    return static_cast<int>(min(static_cast<uint32_t>(id), static_cast<uint32_t>(G)));
  };
  const int per = (M + kNT - 1) / kNT * 64;  // ids per wave, whole rows of lanes
  const int lo = min(wave * per, M), hi = min(lo + per, M);
  int nb = 0, nm = 0;
  for (int i = lo + lane; i < hi; i += 64) {
    const int v = group_of(ids[i]);
    nb += v < g;
    nm += v == g;
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) {
    nb += __shfl_xor(nb, s);
    nm += __shfl_xor(nm, s);
  }
  if (lane == 0) {
    below[wave] = nb;
    mine[wave] = nm;
  }
  __syncthreads();
  int start = 0, at = 0;
#pragma unroll
  for (int w = 0; w < kNW; ++w) {
    start += below[w];
    at += w < wave ? mine[w] : 0;
  }
  if (threadIdx.x == 0) offsets[g] = start;
  if (!order) return;
  at += start;
  for (int i0 = lo; i0 < hi; i0 += 64) {
    const int i = i0 + lane;
    const bool hit = i < hi && group_of(ids[i]) == g;
    const uint64_t m = __ballot(hit);
    if (hit) order[at + __popcll(m & ((uint64_t{1} << lane) - 1))] = i;
    at += __popcll(m);
  }
}

}  // namespace

hipError_t launch_group_rows(int64_t M, int32_t G, const int32_t* ids, int32_t* offsets,
                             int32_t* order, hipStream_t s) {
  group_rows_kernel<<<static_cast<unsigned>(G + 1), kNT, 0, s>>>(
      ids, static_cast<int32_t>(M), G, offsets, M > 0 ? order : nullptr);
  return hipGetLastError();
}

}  // namespace bnn
