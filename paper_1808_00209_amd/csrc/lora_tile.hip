// The matrix-core kernels of the shared binary layer with adapters
// (bnn_bgemm_lora): one pass over x for its sign bits and u = scale (x a^T),
// then binary GEMM tiles whose epilogue adds u b^T.  Both work on positions of
// the order: position p is row order[p] (p itself without an order), and bits
// and u lie by position.  A row's sums are taken in an order that hangs on the
// number of rows (k slices), not on which ones lie beside it.
//
// 8192 rows, 4096 -> 4096, 32 adapters of rank 16, bf16: x pass 30 us for 67 MB
// (20 for x and its signs alone, a 6; 32 where every lane loads the 8 offsets
// it adds, as many bytes through L1 as x), products and epilogue 70-72 (53 for
// the products to bits in the FC kernel; the epilogue 14, all blocks in step, 8
// of stores, 8 of adapters): 98-101 us in runs of one adapter, 245 with the 32
// mixed from row to row and no order.
#include <type_traits>

#include "dtypes.hpp"
#include "expert_plans.hpp"
#include "experts.hpp"
#include "fp4_tile.hpp"
#include "lane_ops.hpp"
#include "lora_parts.hpp"

namespace bnn {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------ x -> bits, u ---
constexpr int kDownNW = 8;             // waves, each an eighth of the block's k groups
constexpr int kDownNT = 64 * kDownNW;
constexpr int kDownRW = 2;             // 16-row tiles per wave
constexpr int kDownRows = 16 * kDownRW;
constexpr int kGroup = 128;            // k per step of a wave: 4 words of sign bits

// A row's 32 consecutive elements as the four lane groups of a 16-row operand
// hold them: lane (q, c) has elements 8 q .. 8 q + 7 of row c.
template <class T>
struct Frag {
  T v[8];
};

// FULL: all 8 elements exist (rows need no alignment beyond the type's);
// otherwise `left` of them do, and the others read 0.
template <bool FULL, class T>
__device__ __forceinline__ Frag<T> load_frag(const T* p, int left) {
  Frag<T> f;
  if constexpr (FULL) {
    __builtin_memcpy(f.v, p, sizeof(f.v));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = i < left ? p[i] : T{};
  }
  return f;
}

// Lane 16 q + I's v in every lane of its row of 16 (DPP row_newbcast, taken by
// the instruction that uses it).
template <int I>
__device__ __forceinline__ float of_row_lane(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x150 + I, 0xF, 0xF, true));
}

// The signs of 8 sums x + off as a byte, element 0 in bit 7.  off's values are
// those of lanes 8 P .. 8 P + 7 of the row.  A sum that is not NaN is above 0
// where its pattern is, as a whole number (it is not -0: off has none); then 0 -
// pattern has the sign bit.
template <int P, class T>
__device__ __forceinline__ uint32_t sign_byte(const Frag<T>& x, float off) {
  uint32_t byte = 0;
  auto add = [&](auto e) {
    constexpr int kE = decltype(e)::value;
    byte = __builtin_amdgcn_alignbit(
        byte, 0u - __float_as_uint(to_f32(x.v[kE]) + of_row_lane<8 * P + kE>(off)), 31);
  };
  add(std::integral_constant<int, 0>{});
  add(std::integral_constant<int, 1>{});
  add(std::integral_constant<int, 2>{});
  add(std::integral_constant<int, 3>{});
  add(std::integral_constant<int, 4>{});
  add(std::integral_constant<int, 5>{});
  add(std::integral_constant<int, 6>{});
  add(std::integral_constant<int, 7>{});
  return byte;
}

__device__ __forceinline__ v4f mma16(const Frag<__bf16>& x, const Frag<__bf16>& y, v4f acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x),
                                                 __builtin_bit_cast(v8bf, y), acc, 0, 0, 0);
}
__device__ __forceinline__ v4f mma16(const Frag<_Float16>& x, const Frag<_Float16>& y, v4f acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x),
                                                __builtin_bit_cast(v8h, y), acc, 0, 0, 0);
}
// fp32: eight products of k = 4, element i of every lane group in the i-th
// (which k goes where does not matter as long as both operands agree).
__device__ __forceinline__ v4f mma16(const Frag<float>& x, const Frag<float>& y, v4f acc) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.v[i], y.v[i], acc, 0, 0, 0);
  return acc;
}

// Block (32 positions, k slice, 16 NR ranks): the sign bits (first rank
// block) and u partial [slice][p][rank].
template <class T, int NR>
__global__ __launch_bounds__(kDownNT) void lora_down_kernel(LoraArgs a, float* __restrict__ u,
                                                            uint32_t* __restrict__ bits,
                                                            int slices) {
  __shared__ float part[kDownNW][kDownRows][16 * NR + 4];
  __shared__ int32_t adapter[kDownRows], adapters;
  __shared__ uint32_t adapter_rows[kDownRows];
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int p0 = blockIdx.x * kDownRows, slice = blockIdx.y, r0 = blockIdx.z * 16 * NR;
  const bool want_bits = blockIdx.z == 0;
  const int kw = (a.K + 31) >> 5;
  const int groups = (a.K + kGroup - 1) / kGroup;

  const T* xr[kDownRW];
  int id[kDownRW];
#pragma unroll
  for (int i = 0; i < kDownRW; ++i) {
    const int p = p0 + 16 * i + c;
    const int row = lora_row(a, p);
    xr[i] = static_cast<const T*>(a.x) + row * a.x_stride + 8 * q;
    id[i] = p < a.M ? lora_adapter(a, row) : -1;
  }
  // The adapters among the block's rows, each with its rows (bit 16 i + c).
  if (wave == 0) {
    uint32_t todo = 0;
#pragma unroll
    for (int i = 0; i < kDownRW; ++i)
      todo |= static_cast<uint32_t>(__ballot(id[i] >= 0) & 0xFFFFu) << (16 * i);
    int n = 0;
    for (; todo; ++n) {
      const int at = __builtin_ctz(todo);
      const int l = __builtin_amdgcn_readlane(at < 16 ? id[0] : id[1], at & 15);
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < kDownRW; ++i)
        m |= static_cast<uint32_t>(__ballot(id[i] == l) & 0xFFFFu) << (16 * i);
      todo &= ~m;
      if (lane == 0) {
        adapter[n] = l;
        adapter_rows[n] = m;
      }
    }
    if (lane == 0) adapters = n;
  }
  typedef Frag<T> Xs[4][kDownRW];
  typedef Frag<T> As[4][NR];
  v4f acc[kDownRW][NR] = {};
  auto load_x = [&](Xs& x, int g, auto full) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < kDownRW; ++i) {
        const int k = g * kGroup + 32 * s;
        x[s][i] = load_frag<decltype(full)::value, T>(xr[i] + k, a.K - k - 8 * q);
      }
  };
  auto load_a = [&](As& w, int d, int g, auto full) {
    const T* ar = static_cast<const T*>(a.a) +
                  static_cast<size_t>(__builtin_amdgcn_readfirstlane(adapter[d])) * a.rank * a.K +
                  8 * q;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = r0 + 16 * n + c;  // (past the last rank: read rank 0, dropped at the end)
      const T* src = ar + static_cast<size_t>(r < a.rank ? r : 0) * a.K;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = g * kGroup + 32 * s;
        w[s][n] = load_frag<decltype(full)::value, T>(src + k, a.K - k - 8 * q);
      }
    }
  };
  // A lane's sums are those of one row: they take an adapter's products where
  // the row is the adapter's, and keep theirs else (as zeros in the product
  // other rows would take 0 x infinity).
  auto multiply = [&](const Xs& x, const As& w, int d) {
    const uint32_t rows = adapter_rows[d];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      v4f sum[kDownRW];
#pragma unroll
      for (int i = 0; i < kDownRW; ++i) sum[i] = acc[i][n];
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < kDownRW; ++i) sum[i] = mma16(w[s][n], x[s][i], sum[i]);
#pragma unroll
      for (int i = 0; i < kDownRW; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][n][e] = (rows >> (16 * i + c)) & 1 ? sum[i][e] : acc[i][n][e];
    }
  };
  // The offsets of a group, an element per lane and load: lane (q, c) has
  // element c % 8 of its q's eight, of the 32 k of step 2 j + c / 8.
  float off[2] = {0.0f, 0.0f};
  auto load_off = [&](int g, auto full) {
    if (!want_bits || !a.offset) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = g * kGroup + 32 * (2 * j + (c >> 3)) + 8 * q + (c & 7);
      off[j] = decltype(full)::value || k < a.K ? a.offset[k] : 0.0f;
    }
  };
  // Elements past K are 0 with offset 0: bit 0.
  auto make_bits = [&](const Xs& x, int g) {
    uint32_t w[kDownRW][4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // -0 to +0; NaN, whose sum reads -1, to an infinity that does as well
      const float o = off[j] == off[j] ? off[j] + 0.0f : -INFINITY;
#pragma unroll
      for (int i = 0; i < kDownRW; ++i) {
        w[i][2 * j] = sign_byte<0>(x[2 * j][i], o) << (24 - 8 * q);
        w[i][2 * j + 1] = sign_byte<1>(x[2 * j + 1][i], o) << (24 - 8 * q);
      }
    }
#pragma unroll
    for (int i = 0; i < kDownRW; ++i) {
      // lane (q, c): word q of row c
      const uint32_t word = or_rows4(w[i][0], w[i][1], w[i][2], w[i][3]);
      const int p = p0 + 16 * i + c, wi = 4 * g + q;
      if (p < a.M && wi < kw) bits[static_cast<size_t>(p) * kw + wi] = word;
    }
  };

  // Whole groups, the next one's x in flight, and up to 16 ranks the next
  // adapter's rows; then what is left of K.
  // (consecutive groups of a wave: 34 us for the 8192 rows below, against 37
  // with the waves' groups interleaved)
  const int per = (groups + slices * kDownNW - 1) / (slices * kDownNW);
  int g = (slice * kDownNW + wave) * per;
  const int end = min(g + per, groups), whole = min(a.K / kGroup, end);
  constexpr bool kAhead = NR == 1;
  Xs x;
  As w;
  if (g < whole) load_x(x, g, std::true_type{});
  __syncthreads();
  const int nd = __builtin_amdgcn_readfirstlane(adapters);
  if (g < whole) {
    if (kAhead && nd) load_a(w, 0, g, std::true_type{});
    for (; g < whole; ++g) {
      Xs next;
      load_off(g, std::true_type{});
      load_x(next, min(g + 1, whole - 1), std::true_type{});
      for (int d = 0; d < nd; ++d) {
        if constexpr (kAhead) {
          As after;
          const bool last = d + 1 == nd;
          load_a(after, last ? 0 : d + 1, last ? min(g + 1, whole - 1) : g, std::true_type{});
          multiply(x, w, d);
          __builtin_memcpy(&w, &after, sizeof(w));
        } else {
          load_a(w, d, g, std::true_type{});
          multiply(x, w, d);
        }
      }
      if (want_bits) make_bits(x, g);
      __builtin_memcpy(&x, &next, sizeof(x));
    }
  }
  if (g < end) {
    load_x(x, g, std::false_type{});
    load_off(g, std::false_type{});
    for (int d = 0; d < nd; ++d) {
      load_a(w, d, g, std::false_type{});
      multiply(x, w, d);
    }
    if (want_bits) make_bits(x, g);
  }
  // The waves' parts of u meet in LDS, added in the waves' order.
#pragma unroll
  for (int i = 0; i < kDownRW; ++i)
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][16 * i + c][16 * n + 4 * q + e] = acc[i][n][e];
  __syncthreads();
  for (int v = tid; v < kDownRows * 16 * NR; v += kDownNT) {
    const int i = v / (16 * NR), r = v % (16 * NR), p = p0 + i;
    if (p >= a.M || r0 + r >= a.rank) continue;
    const int l = lora_adapter(a, lora_row(a, p));
    if (l < 0) continue;
    float sum = part[0][i][r];
#pragma unroll
    for (int w = 1; w < kDownNW; ++w) sum += part[w][i][r];
    u[(static_cast<size_t>(slice) * a.M + p) * a.rank + r0 + r] =
        sum * (a.scale ? a.scale[l] : 1.0f);
  }
}

// --------------------------------------------------------- bits, u -> y ---
struct UpArgs {
  LoraArgs a;
  const float* u;
  const uint32_t* bits;
  uint32_t bits_bytes, w_bytes, tmask;
  int32_t Kw, chunks, slices, wfl;
  uint32_t cols;
  int32_t row_tiles;
};

template <class T, class Y, int PT>
__global__ __launch_bounds__(kTileNT, 2) void lora_up_kernel(UpArgs g) {
  extern __shared__ v4i act[];
  const LoraArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, c = lane & 31;
  // Block b runs on XCD b mod 8: an XCD takes consecutive tiles, the outputs
  // fastest, so that its L2 serves a row tile to all of them.
  const uint32_t tile = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  const int rt = static_cast<int>(tile / g.cols);
  if (rt >= g.row_tiles) return;
  const int ft = static_cast<int>(tile - static_cast<uint32_t>(rt) * g.cols);
  const int wp = 4 >> g.wfl;
  const int m00 = rt * wp * PT * 32;
  const int f0 = (ft << (6 + g.wfl)) + (wave & ((1 << g.wfl) - 1)) * 64;

  TileLoop t;
  t.ra = tile_rsrc(g.bits, g.bits_bytes);
  t.rb = tile_rsrc(a.w, g.w_bytes);
#pragma unroll
  for (int tf = 0; tf < 2; ++tf)
    t.woff[tf] = (static_cast<uint32_t>(f0 + 32 * tf + c) * g.Kw + 4 * h) * 4;
  t.K = a.K;
  t.Kw = g.Kw;
  t.chunks = g.chunks;
  t.tmask = g.tmask;
  t.wpi = wave >> g.wfl;
  v16f acc[2][PT];
#pragma unroll
  for (int tf = 0; tf < 2; ++tf)
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) acc[tf][pt] = v16f{};
  tile_loop<PT>(acc, act, t, [&] {
    return (static_cast<uint32_t>(min(m00 + (tid >> 1), a.M - 1)) * g.Kw + 4 * (tid & 1)) * 4;
  });

  // y = alpha S + u b^T, 32 rows after another.  u b^T takes 16 ranks at a time,
  // and of these one adapter of the rows after another, in sums of its own (S
  // is exact: so alpha S is rounded once, whatever the adapters add up).  While
  // one such step multiplies, the next one's values are loaded, the next rows'
  // first step among them.  A row's outputs leave through LDS (a region per
  // wave) as one run.
  constexpr int kV = 16 / sizeof(Y);    // outputs per 16-byte store
  constexpr int kLanes = 64 / kV;       // lanes per row
  constexpr int kStride = 64 + kV;      // LDS outputs per row of 64
  constexpr int kRegion = 33 * 68 * 4;  // LDS bytes per wave
  static_assert(32 * kStride * sizeof(Y) + 64 * sizeof(float) <= kRegion, "rows and alphas");
  Y* ts = reinterpret_cast<Y*>(reinterpret_cast<char*>(act) + wave * kRegion);
  float* al = reinterpret_cast<float*>(ts + 32 * kStride);  // alpha of the wave's 64 outputs
  const bool wide = a.N % kV == 0;
  al[lane] = f0 + lane < a.N && a.alpha ? a.alpha[f0 + lane] : 1.0f;
  const int base = m00 + t.wpi * PT * 32 + c;
  int row[PT], id[PT];
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) row[pt] = lora_row(a, base + 32 * pt);
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) id[pt] = base + 32 * pt < a.M ? lora_adapter(a, row[pt]) : -1;

  RawB<T> nb[2];
  float nu[8];
  auto fetch_u = [&](int mine, int p, int r) {  // (mine < 0: other values)
    const int rr = r + 8 * h;
    const float* src =
        g.u + (mine >= 0 && rr < a.rank ? static_cast<size_t>(p) * a.rank + rr : size_t{0});
    __builtin_memcpy(nu, __builtin_assume_aligned(src, 16), sizeof(nu));
    for (int s = 1; s < g.slices; ++s) {
      float w[8];
      __builtin_memcpy(
          w, __builtin_assume_aligned(src + static_cast<size_t>(s) * a.M * a.rank, 16), sizeof(w));
#pragma unroll
      for (int e = 0; e < 8; ++e) nu[e] += w[e];
    }
  };
  auto fetch_b = [&](int tf, int l, int r) {
    nb[tf] = load_b<T>(a, l, f0 + 32 * tf + c, r + 8 * h);
  };
  auto waiting = [&](int pt) { return static_cast<uint32_t>(__ballot(id[pt] >= 0)); };
  // The first step of rows pt.
  auto fetch_first = [&](int pt, uint32_t rows) {
    const int l = __builtin_amdgcn_readlane(id[pt], __builtin_ctz(rows));
    fetch_b(0, l, 0);
    fetch_b(1, l, 0);
    fetch_u(id[pt], base + 32 * pt, 0);
  };
  if (const uint32_t rows = waiting(0)) fetch_first(0, rows);
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) {
    asm volatile("" ::: "memory");  // (no loads of later rows up here: registers)
    const int np = pt + 1 < PT ? pt + 1 : pt;
    const uint32_t rows = waiting(pt), next_rows = np > pt ? waiting(np) : 0u;
    v16f low[2] = {};
    if (!rows && next_rows) fetch_first(np, next_rows);
    for (int r = 0; rows && r < a.rank; r += 16) {
      v8bf u[3];
      split_frag<3>(nu, r + 8 * h < a.rank, u);
      for (uint32_t todo = rows; todo;) {
        const int l = __builtin_amdgcn_readlane(id[pt], __builtin_ctz(todo));
        todo &= ~static_cast<uint32_t>(__ballot(id[pt] == l));
        // The next step: another adapter, 16 ranks more, or the next rows.
        const bool last = !todo && r + 16 >= a.rank;
        const uint32_t from = todo ? todo : last ? next_rows : rows;
        const int whose = last ? id[np] : id[pt];
        const int nr = todo ? r : last ? 0 : r + 16;
        const int nl = from ? __builtin_amdgcn_readlane(whose, __builtin_ctz(from)) : 0;
#pragma unroll
        for (int tf = 0; tf < 2; ++tf) {
          v8bf b[kParts<T>];
          split_b<T>(nb[tf], f0 + 32 * tf + c < a.N && r + 8 * h < a.rank, b);
          if (from) fetch_b(tf, nl, nr);
          if (tf == 1 && from && !todo) fetch_u(whose, base + 32 * (last ? np : pt), nr);
          add_rows<T>(low[tf], b, u, id[pt] == l);
          // (one tile's sums at a time: both take registers that spill)
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    // Register e of a tile holds output 8 (e / 4) + 4 h + e % 4 of row c.
#pragma unroll
    for (int tf = 0; tf < 2; ++tf)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int n = 32 * tf + 2 * e + 4 * h;
        float f[4];
        __builtin_memcpy(f, __builtin_assume_aligned(&al[n], 16), sizeof(f));
        Y y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = from_f32<Y>(fmaf(acc[tf][pt][e + i], f[i], low[tf][e + i]));
        __builtin_memcpy(__builtin_assume_aligned(&ts[c * kStride + n], sizeof(y)), y, sizeof(y));
      }
#pragma unroll
    for (int o = 0; o < 32; o += 64 / kLanes) {
      const int i = o + lane / kLanes, col = kV * (lane % kLanes), n = f0 + col;
      const int m = __shfl(row[pt], i);
      Y v[kV];
      __builtin_memcpy(v, __builtin_assume_aligned(&ts[i * kStride + col], 16), sizeof(v));
      if (base - c + 32 * pt + i < a.M) {
        Y* dst = static_cast<Y*>(a.y) + static_cast<size_t>(m) * a.N + n;
        if (wide) {
          if (n < a.N) __builtin_memcpy(__builtin_assume_aligned(dst, 16), v, 16);
        } else {
#pragma unroll
          for (int e = 0; e < kV; ++e)
            if (n + e < a.N) dst[e] = v[e];
        }
      }
    }
  }
}

size_t u_bytes(int64_t M, int32_t K, int32_t rank) {
  return static_cast<size_t>(lora_down_slices(M, K, rank)) * M * rank * sizeof(float);
}

}  // namespace

size_t lora_tile_workspace(int64_t M, int32_t K, int32_t rank) {
  return (static_cast<size_t>(lora_u_rows(M, K, rank)) * rank + static_cast<size_t>(M) * words_of(K)) *
         4;
}

bool lora_tile_supported(const LoraArgs& a) {
  return static_cast<int64_t>(a.M) * words_of(a.K) * 4 < (int64_t{1} << 32) - 64;
}

hipError_t launch_lora_tile(const LoraArgs& a, hipStream_t s) {
  UpArgs g;
  g.a = a;
  float* u = static_cast<float*>(a.ws);
  uint32_t* bits = reinterpret_cast<uint32_t*>(static_cast<char*>(a.ws) +
                                               u_bytes(a.M, a.K, a.rank));
  g.u = u;
  g.bits = bits;
  g.Kw = static_cast<int32_t>(words_of(a.K));
  g.bits_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.M) * g.Kw * 4);
  g.w_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.N) * g.Kw * 4);
  g.tmask = tail_mask(a.K);
  g.chunks = (g.Kw + 7) / 8;
  const bool by_rows = lora_down_by_rows(a.M, a.rank);
  g.slices = lora_down_slices(a.M, a.K, a.rank);
  const TileShape shape = lora_shape(a.M, a.N, g.chunks);
  g.wfl = shape.wfl;
  g.cols = static_cast<uint32_t>((a.N + shape.outputs() - 1) / shape.outputs());
  g.row_tiles = (a.M + shape.rows() - 1) / shape.rows();
  const unsigned grid =
      static_cast<unsigned>((static_cast<int64_t>(g.cols) * g.row_tiles + 7) / 8 * 8);
  static_assert(kTileLds >= size_t{4} * 33 * 68 * 4, "the output tiles fit");
  with_real_type(a.dtype, [&](auto v) {
    using T = decltype(v);
    const unsigned bx = static_cast<unsigned>((a.M + kDownRows - 1) / kDownRows);
    const unsigned by = static_cast<unsigned>(g.slices);
    if (by_rows)
      launch_lora_down_rows(a, u, bits, s);
    else if (a.rank <= 16)
      lora_down_kernel<T, 1><<<dim3(bx, by, 1), kDownNT, 0, s>>>(a, u, bits, g.slices);
    else if (a.rank <= 32)
      lora_down_kernel<T, 2><<<dim3(bx, by, 1), kDownNT, 0, s>>>(a, u, bits, g.slices);
    else
      lora_down_kernel<T, 4><<<dim3(bx, by, static_cast<unsigned>((a.rank + 63) / 64)), kDownNT, 0,
                               s>>>(a, u, bits, g.slices);
    if (lora_up_skinny(a.M, a.N)) {
      launch_lora_up_skinny(a, u, bits, g.slices, s);
      return;
    }
    with_real_type(a.out_dtype, [&](auto y) {
      using Y = decltype(y);
      switch (shape.pt) {
        case 4: lora_up_kernel<T, Y, 4><<<grid, kTileNT, kTileLds, s>>>(g); break;
        case 2: lora_up_kernel<T, Y, 2><<<grid, kTileNT, kTileLds, s>>>(g); break;
        default: lora_up_kernel<T, Y, 1><<<grid, kTileNT, kTileLds, s>>>(g); break;
      }
    });
  });
  return hipGetLastError();
}

}  // namespace bnn
