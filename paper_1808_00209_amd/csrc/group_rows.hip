// Rows in the order of their group (bnn_group_rows): a stable counting sort.
// No atomics decide an order, so it is that of the rows.
//
// Up to 16384 rows, one launch: block g belongs to group g, block G to the
// rows of no group.  Every block reads all ids, for the number of rows of
// lower groups, where its own begin, and for its own rows, whose places it
// keeps as bit masks in LDS; then it writes them.
//
// More rows, two launches: chunks of rows are counted by group into the
// workspace; then every chunk's block adds up the counts before it and places
// its rows.  131072 rows, 256 groups: 35 us in the first form (every compute
// unit passes over all ids), 11 us in the second.
#include "experts.hpp"
#include "group_tiles.hpp"

namespace bnn {
namespace {

// An id outside [0, G) counts as group G.
__device__ __forceinline__ int group_of(int32_t id, int32_t G) {
  return static_cast<int>(min(static_cast<uint32_t>(id), static_cast<uint32_t>(G)));
}

// LDS operations of a wave complete in their order: this keeps the compiler
// from moving them, for values that other lanes of the wave wrote.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------- one launch ---
constexpr int kOneRows = 16384;  // most rows
constexpr int kOneNW = 16;       // most waves
constexpr int kUnroll = 8;       // loads in flight

__global__ __launch_bounds__(64 * kOneNW) void group_rows_kernel(const int32_t* __restrict__ ids,
                                                                 int32_t M, int32_t G,
                                                                 int32_t* __restrict__ offsets,
                                                                 int32_t* __restrict__ order) {
  __shared__ uint64_t masks[kOneRows / 64 + kOneNW];  // [waves][64-row pieces of a wave]
  __shared__ int32_t below[kOneNW], mine[kOneNW];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int nw = static_cast<int>(blockDim.x) >> 6;
  const int g = blockIdx.x;
  // A wave takes a contiguous part of the ids.
  const int pieces = (M + 63) / 64;
  const int per = (pieces + nw - 1) / nw;
  const int lo = min(wave * per, pieces), hi = min(lo + per, pieces);
  uint64_t* own = masks + wave * per;
  int nb = 0, nm = 0;
  for (int p = lo; p < hi; p += kUnroll) {
    int v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = ids[min(64 * (p + u) + lane, M - 1)];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const bool in = p + u < hi && 64 * (p + u) + lane < M;
      const int q = group_of(v[u], G);
      nb += in && q < g ? 1 : 0;
      const uint64_t m = __ballot(in && q == g);
      nm += __popcll(m);
      if (lane == u && p + u < hi) own[p + u - lo] = m;
    }
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) nb += __shfl_xor(nb, s);
  if (lane == 0) {
    below[wave] = nb;
    mine[wave] = nm;
  }
  __syncthreads();
  int start = 0, at = 0;
  for (int w = 0; w < nw; ++w) {
    start += below[w];
    at += w < wave ? mine[w] : 0;
  }
  if (threadIdx.x == 0) offsets[g] = start;
  at += start;
  wave_order();
  // A lane per piece: its place among the wave's pieces, then its rows.
  for (int p = 0; p < hi - lo; p += 64) {
    uint64_t m = p + lane < hi - lo ? own[p + lane] : 0;
    const int n = __popcll(m), sum = wave_scan(n);
    int to = at + sum - n;
    for (; m; m &= m - 1) order[to++] = 64 * (lo + p + lane) + __builtin_ctzll(m);
    at += __builtin_amdgcn_readlane(sum, 63);
  }
}

// ------------------------------------------------------------ two launches ---
constexpr int kNT = 1024;
constexpr int kNW = kNT / 64;
constexpr int kRounds = 2;                 // rows per thread and step
constexpr int kStep = kRounds * kNT;       // rows per step of a block
constexpr int kMaxChunks = 128;
constexpr int kBins = BNN_MAX_EXPERTS + 1;

// Steps of kStep rows per chunk, so that there are at most kMaxChunks.
__host__ __device__ inline int chunk_steps(int32_t M) {
  const int steps = (M + kStep - 1) / kStep;
  return (steps + kMaxChunks - 1) / kMaxChunks;
}
inline int chunk_count(int32_t M) {
  const int rows = chunk_steps(M) * kStep;
  return (M + rows - 1) / rows;
}

// counts[chunk][g]: rows of the chunk in group g (G: none).
__global__ __launch_bounds__(kNT) void group_count_kernel(const int32_t* __restrict__ ids,
                                                          int32_t M, int32_t G, int32_t steps,
                                                          int32_t* __restrict__ counts) {
  __shared__ int32_t bins[kBins];
  for (int g = threadIdx.x; g <= G; g += kNT) bins[g] = 0;
  __syncthreads();
  const int64_t first = static_cast<int64_t>(blockIdx.x) * steps * kStep;
  for (int s = 0; s < steps; ++s) {
    int v[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int64_t i = first + s * kStep + r * kNT + threadIdx.x;
      v[r] = i < M ? group_of(ids[i], G) : -1;
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (v[r] >= 0) atomicAdd(&bins[v[r]], 1);
  }
  __syncthreads();
  for (int g = threadIdx.x; g <= G; g += kNT)
    counts[static_cast<size_t>(blockIdx.x) * (G + 1) + g] = bins[g];
}

__global__ __launch_bounds__(kNT) void group_place_kernel(const int32_t* __restrict__ ids,
                                                          int32_t M, int32_t G, int32_t steps,
                                                          int32_t id_bits,
                                                          const int32_t* __restrict__ counts,
                                                          int32_t* __restrict__ offsets,
                                                          int32_t* __restrict__ order) {
  __shared__ int32_t base[kBins];           // where the group's next row goes
  __shared__ uint16_t wcnt[kNW][kBins + 1]; // rows of the step by wave and group
  __shared__ int32_t sums[kNW];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int chunk = blockIdx.x, chunks = gridDim.x;
  // Group tid (1024 groups and the rows of none: the last one is what is left).
  int before = 0, total = 0;
  if (tid <= G) {
#pragma unroll 8
    for (int c = 0; c < chunks; ++c) {
      const int n = counts[static_cast<size_t>(c) * (G + 1) + tid];
      before += c < chunk ? n : 0;
      total += n;
    }
  }
  int last_before = 0;  // of group 1024, where there is one
  if (G == kNT && tid == 0)
    for (int c = 0; c < chunk; ++c) last_before += counts[static_cast<size_t>(c) * (G + 1) + kNT];
  const int scan = wave_scan(total);
  if (lane == 63) sums[wave] = scan;
  __syncthreads();
  int start = scan - total, all = 0;
  for (int w = 0; w < kNW; ++w) {
    start += w < wave ? sums[w] : 0;
    all += sums[w];
  }
  if (tid <= G) {
    base[tid] = start + before;
    if (chunk == 0) offsets[tid] = start;
  }
  if (G == kNT && tid == 0) {
    base[kNT] = all + last_before;
    if (chunk == 0) offsets[kNT] = all;
  }
  const int64_t first = static_cast<int64_t>(chunk) * steps * kStep;
  for (int s = 0; s < steps; ++s) {
    // A wave's rows are consecutive: 64 kRounds of the step's.
    const int64_t i0 = first + s * kStep + wave * (64 * kRounds) + lane;
    for (int g = lane; g <= G; g += 64) wcnt[wave][g] = 0;
    int v[kRounds], rel[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) v[r] = i0 + 64 * r < M ? group_of(ids[i0 + 64 * r], G) : -1;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      wave_order();
      // The lanes of the same group, by a ballot per bit of the group.
      uint64_t same = __ballot(v[r] >= 0);
      for (int b = 0; b < id_bits; ++b) {
        const bool on = (v[r] >> b) & 1;
        const uint64_t m = __ballot(on);
        same &= on ? m : ~m;
      }
      const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
      rel[r] = 0;
      if (v[r] >= 0) {
        rel[r] = wcnt[wave][v[r]] + rank;
        if (rank == 0) wcnt[wave][v[r]] += static_cast<uint16_t>(__popcll(same));
      }
    }
    __syncthreads();
    // Counts become the rows of the earlier waves; base moves on below.
    int moved[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int g = tid + k * kNT;
      if (g > G) continue;
      int sum = 0;
      for (int w = 0; w < kNW; ++w) {
        const int n = wcnt[w][g];
        wcnt[w][g] = static_cast<uint16_t>(sum);
        sum += n;
      }
      moved[k] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (v[r] >= 0)
        order[min(base[v[r]] + wcnt[wave][v[r]] + rel[r], M - 1)] = static_cast<int>(i0 + 64 * r);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (tid + k * kNT <= G) base[tid + k * kNT] += moved[k];
  }
}

}  // namespace

size_t group_rows_workspace(int64_t M, int32_t G) {
  if (M <= kOneRows) return 0;
  // (the chunks of M rows or of any fewer: longer ones are fewer again)
  const int64_t steps = (M + kStep - 1) / kStep;
  return static_cast<size_t>(steps < kMaxChunks ? steps : kMaxChunks) * (G + 1) * sizeof(int32_t);
}

hipError_t launch_group_rows(int64_t M, int32_t G, const int32_t* ids, int32_t* offsets,
                             int32_t* order, void* ws, hipStream_t s) {
  const int32_t m = static_cast<int32_t>(M);
  if (m <= kOneRows) {
    // Waves: 16, or as many as have 8 pieces of 64 rows each.
    int nw = (m + 511) / 512;
    nw = nw < 1 ? 1 : nw > kOneNW ? kOneNW : nw;
    group_rows_kernel<<<static_cast<unsigned>(G + 1), 64 * nw, 0, s>>>(ids, m, G, offsets, order);
    return hipGetLastError();
  }
  const int steps = chunk_steps(m);
  const unsigned chunks = static_cast<unsigned>(chunk_count(m));
  int bits = 0;
  while ((1 << bits) <= G) ++bits;  // group G is an id too
  int32_t* counts = static_cast<int32_t*>(ws);
  group_count_kernel<<<chunks, kNT, 0, s>>>(ids, m, G, steps, counts);
  group_place_kernel<<<chunks, kNT, 0, s>>>(ids, m, G, steps, bits, counts, offsets, order);
  return hipGetLastError();
}

}  // namespace bnn
