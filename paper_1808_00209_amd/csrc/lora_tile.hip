// The matrix-core kernels of the shared binary layer with adapters
// (bnn_bgemm_lora): one pass over x for its sign bits and u = scale (x a^T),
// then binary GEMM tiles whose epilogue adds u b^T.  Both work on positions of
// the order: position p is row order[p] (p itself without an order), and bits
// and u lie by position.  A row's sums are taken in an order that does not
// hang on the rows beside it.
#include "dtypes.hpp"
#include "experts.hpp"
#include "fp4_tile.hpp"
#include "lane_ops.hpp"

namespace bnn {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int row_of(const LoraArgs& a, int p) {
  p = min(p, a.M - 1);
  return a.order ? static_cast<int>(min(static_cast<uint32_t>(a.order[p]),
                                        static_cast<uint32_t>(a.M - 1)))
                 : p;
}

// The adapter of a row, -1 for none.
__device__ __forceinline__ int adapter_of(const LoraArgs& a, int row) {
  const int l = a.ids[row];
  return l >= 0 && l < a.adapters ? l : -1;
}

// ------------------------------------------------------------ x -> bits, u ---
constexpr int kDownNW = 8;             // waves, each an eighth of the block's k groups
constexpr int kDownNT = 64 * kDownNW;
constexpr int kDownRW = 2;             // 16-row tiles per wave
constexpr int kDownRows = 16 * kDownRW;
constexpr int kGroup = 128;            // k per step of a wave: 4 words of sign bits

// A row's 32 consecutive elements as the four lane groups of a 16-row operand
// hold them: lane (q, c) has elements 8 q .. 8 q + 7 of row c.  `left`: the
// elements from 8 q on that exist (rows need no alignment beyond the type's).
template <class T>
struct Frag {
  T v[8];
};

template <class T>
__device__ __forceinline__ Frag<T> load_frag(const T* p, int left) {
  Frag<T> f;
  if (left >= 8) {
    __builtin_memcpy(f.v, p, sizeof(f.v));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = i < left ? p[i] : T{};
  }
  return f;
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
    const int row = row_of(a, p);
    xr[i] = static_cast<const T*>(a.x) + row * a.x_stride + 8 * q;
    id[i] = p < a.M ? adapter_of(a, row) : -1;
  }
  v4f acc[kDownRW][NR] = {};
  // One pass over the slice per adapter among the block's rows (mostly one);
  // the first pass, with or without an adapter, makes the sign bits.
  uint32_t todo = 0;  // bit 16 i + c: the row still waits for its adapter
#pragma unroll
  for (int i = 0; i < kDownRW; ++i)
    todo |= static_cast<uint32_t>(__ballot(id[i] >= 0) & 0xFFFFu) << (16 * i);
  for (bool first = true; first || todo; first = false) {
    int l = -1;
    if (todo) {
      const int at = __builtin_ctz(todo);
      l = __builtin_amdgcn_readlane(at < 16 ? id[0] : id[1], at & 15);
    } else if (!want_bits) {
      break;
    }
    bool mine[kDownRW];
#pragma unroll
    for (int i = 0; i < kDownRW; ++i) {
      mine[i] = l >= 0 && id[i] == l;
      todo &= ~(static_cast<uint32_t>(__ballot(mine[i]) & 0xFFFFu) << (16 * i));
    }
    const T* ar = static_cast<const T*>(a.a) +
                  (static_cast<size_t>(max(l, 0)) * a.rank + r0 + c) * a.K + 8 * q;
    for (int g = slice * kDownNW + wave; g < groups; g += slices * kDownNW) {
      Frag<T> x[4][kDownRW];
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int i = 0; i < kDownRW; ++i) {
          const int k = g * kGroup + 32 * s;
          x[s][i] = load_frag<T>(xr[i] + k, a.K - k - 8 * q);
        }
      if (l >= 0) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int k = g * kGroup + 32 * s;
          Frag<T> xm[kDownRW];
#pragma unroll
          for (int i = 0; i < kDownRW; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) xm[i].v[e] = mine[i] ? x[s][i].v[e] : T{};
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const Frag<T> w = load_frag<T>(ar + static_cast<size_t>(16 * n) * a.K + k,
                                           r0 + 16 * n + c < a.rank ? a.K - k - 8 * q : 0);
#pragma unroll
            for (int i = 0; i < kDownRW; ++i) acc[i][n] = mma16(w, xm[i], acc[i][n]);
          }
        }
      }
      if (first && want_bits) {
        float off[4][8];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int k = g * kGroup + 32 * s + 8 * q + e;
            off[s][e] = a.offset && k < a.K ? a.offset[k] : 0.0f;
          }
#pragma unroll
        for (int i = 0; i < kDownRW; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            uint32_t byte = 0;  // (elements past K are 0 with offset 0: bit 0)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              byte = 2 * byte + (to_f32(x[s][i].v[e]) + off[s][e] > 0.0f ? 1u : 0u);
            w[s] = byte << (24 - 8 * q);
          }
          const uint32_t word = or_rows4(w[0], w[1], w[2], w[3]);  // lane (q, c): word q
          const int p = p0 + 16 * i + c, wi = 4 * g + q;
          if (p < a.M && wi < kw) bits[static_cast<size_t>(p) * kw + wi] = word;
        }
      }
    }
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
    const int l = adapter_of(a, row_of(a, p));
    if (l < 0) continue;
    float sum = part[0][i][r];
#pragma unroll
    for (int w = 1; w < kDownNW; ++w) sum += part[w][i][r];
    u[(static_cast<size_t>(slice) * a.M + p) * a.rank + r0 + r] =
        sum * (a.scale ? a.scale[l] : 1.0f);
  }
}

// --------------------------------------------------------- bits, u -> y ---
// Parts of a value on the bf16 matrix cores: 1 (bf16), 2 (fp16: 11 significant
// bits) or 3 (fp32), each product of u's three parts and these exact.
template <class T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
template <>
constexpr int kParts<_Float16> = 2;

struct UpArgs {
  LoraArgs a;
  const float* u;
  const uint32_t* bits;
  uint32_t bits_bytes, w_bytes, tmask;
  int32_t Kw, chunks, slices, wfl;
  uint32_t cols;
  int32_t row_tiles;
};

// Eight values of u (or b) as bf16 operands, one per part.
template <int P>
__device__ __forceinline__ void split_frag(const float (&v)[8], bool keep, v8bf (&out)[P]) {
  uint16_t b[3][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const Split3 s = split3(keep ? v[e] : 0.0f);
    b[0][e] = bf16_bits(s.p0);
    b[1][e] = bf16_bits(s.p1);
    b[2][e] = bf16_bits(s.p2);
  }
#pragma unroll
  for (int i = 0; i < P; ++i) out[i] = bf16x8(b[i]);
}

// Lane (h, c)'s share of 16 ranks of output row n: b[l][n][16 rc + 8 h ..],
// 0 past the rank or N.
template <class T>
__device__ __forceinline__ void load_b(const LoraArgs& a, int l, int n, int r,
                                       v8bf (&out)[kParts<T>]) {
  const bool in = n < a.N && r < a.rank;
  const T* src = static_cast<const T*>(a.b) +
                 (in ? (static_cast<size_t>(l) * a.N + n) * a.rank + r : size_t{0});
  T v[8];
  __builtin_memcpy(v, __builtin_assume_aligned(src, sizeof(v) > 16 ? 16 : sizeof(v)), sizeof(v));
  if constexpr (kParts<T> == 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = in ? v[e] : T{};
    __builtin_memcpy(&out[0], v, sizeof(v));
  } else {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = to_f32(v[e]);
    split_frag<kParts<T>>(f, in, out);
  }
}

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

  // y = alpha S + u b^T, one 32 x 32 tile after another; u b^T by 16 ranks at a
  // time and one adapter of the tile's rows after another, the rows of other
  // adapters entering as zeros, in sums of its own (S is exact: so alpha S is
  // rounded once, whatever the adapters add up).  A row's outputs leave through
  // LDS (a region per wave: 32 rows x 64 outputs) as one run.
  constexpr int kStride = 68;  // LDS words per row
  float* ts = reinterpret_cast<float*>(act) + wave * (32 * kStride);
  constexpr int kV = 16 / sizeof(Y);  // outputs per 16-byte store
  constexpr int kLanes = 64 / kV;     // lanes per row
  const bool wide = a.N % kV == 0;
  const __amdgpu_buffer_rsrc_t ral = tile_rsrc(a.alpha, a.alpha ? a.N * 4 : 0);
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) {
    asm volatile("" ::: "memory");  // (no loads of later tiles up here: registers)
    const int p0 = m00 + (t.wpi * PT + pt) * 32, p = p0 + c;
    const int id = p < a.M ? adapter_of(a, row_of(a, p)) : -1;
#pragma unroll
    for (int tf = 0; tf < 2; ++tf) {
      uint32_t todo = static_cast<uint32_t>(__ballot(id >= 0));
      v16f low = {};
      while (todo) {
        const int l = __builtin_amdgcn_readlane(id, __builtin_ctz(todo));
        todo &= ~static_cast<uint32_t>(__ballot(id == l));
        for (int r = 0; r < a.rank; r += 16) {
          const int rr = r + 8 * h;
          v8bf b[kParts<T>];
          load_b<T>(a, l, f0 + 32 * tf + c, rr, b);
          const bool mine = id == l && rr < a.rank;
          float v[8] = {};
          for (int s = 0; s < g.slices; ++s) {
            const float* src =
                g.u + (mine ? (static_cast<size_t>(s) * a.M + p) * a.rank + rr : size_t{0});
            float w[8];
            __builtin_memcpy(w, __builtin_assume_aligned(src, 16), sizeof(w));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
          }
          v8bf uf[3];
          split_frag<3>(v, mine, uf);
#pragma unroll
          for (int i = kParts<T> - 1; i >= 0; --i)
#pragma unroll
            for (int j = 2; j >= 0; --j)
              if (i + j < 4)
                low = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[i], uf[j], low, 0, 0, 0);
        }
      }
      // Register e of a tile holds output 8 (e / 4) + 4 h + e % 4 (past N: 0).
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const v4i v = tile_load4(ral, (f0 + 32 * tf + 2 * e + 4 * h) * 4, 0);
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = acc[tf][pt][e + i] * (a.alpha ? __int_as_float(v[i]) : 1.0f) + low[e + i];
        *reinterpret_cast<float4*>(&ts[c * kStride + 32 * tf + 2 * e + 4 * h]) =
            float4{y[0], y[1], y[2], y[3]};
      }
    }
#pragma unroll
    for (int o = 0; o < 32; o += 64 / kLanes) {
      const int i = o + lane / kLanes, col = kV * (lane % kLanes), n = f0 + col;
      Y v[kV];
#pragma unroll
      for (int e = 0; e < kV; ++e) v[e] = from_f32<Y>(ts[i * kStride + col + e]);
      if (p0 + i < a.M) {
        Y* dst = static_cast<Y*>(a.y) + static_cast<size_t>(row_of(a, p0 + i)) * a.N + n;
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

// k slices of the down pass: enough blocks to fill the chip at few rows, at
// least one group of 128 k for every wave.
int down_slices(int64_t M, int32_t K, int32_t rank) {
  const int64_t blocks = (M + kDownRows - 1) / kDownRows * ((rank + 63) / 64);
  const int64_t most = (K + kGroup * kDownNW - 1) / (kGroup * kDownNW);
  const int64_t want = (512 + blocks - 1) / blocks;
  return static_cast<int>(want < most ? want : most);
}

size_t u_bytes(int64_t M, int32_t K, int32_t rank) {
  return static_cast<size_t>(down_slices(M, K, rank)) * M * rank * sizeof(float);
}

}  // namespace

size_t lora_tile_workspace(int64_t M, int32_t K, int32_t rank) {
  return M == 0 ? 0 : u_bytes(M, K, rank) + static_cast<size_t>(M) * words_of(K) * 4;
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
  g.slices = down_slices(a.M, a.K, a.rank);
  g.wfl = a.N > 128 ? 2 : a.N > 64 ? 1 : 0;
  int pt = a.M > 64 ? 4 : a.M > 32 ? 2 : 1;
  pt = pt < (1 << g.wfl) ? pt : 1 << g.wfl;
  const int rows = (4 >> g.wfl) * pt * 32;
  g.cols = static_cast<uint32_t>((a.N + (64 << g.wfl) - 1) / (64 << g.wfl));
  g.row_tiles = (a.M + rows - 1) / rows;
  const unsigned grid =
      static_cast<unsigned>((static_cast<int64_t>(g.cols) * g.row_tiles + 7) / 8 * 8);
  static_assert(kTileLds >= size_t{4} * 32 * 68 * 4, "the output tiles fit");
  with_real_type(a.dtype, [&](auto v) {
    using T = decltype(v);
    const unsigned bx = static_cast<unsigned>((a.M + kDownRows - 1) / kDownRows);
    const unsigned by = static_cast<unsigned>(g.slices);
    if (a.rank <= 16)
      lora_down_kernel<T, 1><<<dim3(bx, by, 1), kDownNT, 0, s>>>(a, u, bits, g.slices);
    else if (a.rank <= 32)
      lora_down_kernel<T, 2><<<dim3(bx, by, 1), kDownNT, 0, s>>>(a, u, bits, g.slices);
    else
      lora_down_kernel<T, 4><<<dim3(bx, by, static_cast<unsigned>((a.rank + 63) / 64)), kDownNT, 0,
                               s>>>(a, u, bits, g.slices);
    with_real_type(a.out_dtype, [&](auto y) {
      using Y = decltype(y);
      switch (pt) {
        case 4: lora_up_kernel<T, Y, 4><<<grid, kTileNT, kTileLds, s>>>(g); break;
        case 2: lora_up_kernel<T, Y, 2><<<grid, kTileNT, kTileLds, s>>>(g); break;
        default: lora_up_kernel<T, Y, 1><<<grid, kTileNT, kTileLds, s>>>(g); break;
      }
    });
  });
  return hipGetLastError();
}

}  // namespace bnn
