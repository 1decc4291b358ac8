// The shared binary layer with adapters (bnn_bgemm_lora) for few rows: a wave
// per row and rank component for u = scale (x a^T), one more per row for its
// sign bits, then 32 x 32 tiles of fp4_skinny.hpp that add u b^T, the adapters
// among a tile's rows dealt out to its waves.  Bits and u lie by position of
// the order.  The time is that of reading the weights and the adapters of the
// rows, and of two launches' chains of loads.  32 rows, 4096 -> 4096, 28
// adapters of rank 16, bf16: 6 + 8 us for 10 MB; on the larger tiles' kernels 64.
#include "dtypes.hpp"
#include "experts.hpp"
#include "fp4_skinny.hpp"
#include "lane_ops.hpp"
#include "lora_parts.hpp"

namespace bnn {
namespace {

// ------------------------------------------------------------ x -> bits, u ---
constexpr int kNT = 256;
constexpr int kNW = kNT / 64;
constexpr int kAdapters = 4;  // adapters whose rows of b are in flight

// 8 elements from p on, of which `left` exist (the others read 0).
template <class T>
__device__ __forceinline__ void load8(T (&v)[8], const T* p, int left) {
  if (left >= 8) {
    __builtin_memcpy(v, p, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : T{};
  }
}

// Block (position, kNW jobs): job 0 the sign bits, job 1 + r component r of u.
template <class T>
__global__ __launch_bounds__(kNT) void lora_down_rows_kernel(LoraArgs a, float* __restrict__ u,
                                                             uint32_t* __restrict__ bits) {
  const int p = blockIdx.x, lane = threadIdx.x & 63;
  const int job = __builtin_amdgcn_readfirstlane(blockIdx.y * kNW + (threadIdx.x >> 6));
  const int r = job - 1;
  if (r >= a.rank) return;
  const int row = lora_row(a, p);
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  constexpr int kAhead = 4;  // 512-element pieces in flight (eight: no quicker)
  if (job == 0) {
    const int kw = (a.K + 31) >> 5;
    for (int k0 = 0; k0 < a.K; k0 += 512 * kAhead) {
      T v[kAhead][8];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int k = k0 + 512 * i + 8 * lane;
        if (k0 + 512 * i < a.K) load8(v[i], x + k, a.K - k);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (k0 + 512 * i >= a.K) break;  // (uniform: all lanes take part below)
        const int k = k0 + 512 * i + 8 * lane;
        float off[8] = {};
        if (a.offset) load8(off, a.offset + k, a.K - k);
        uint32_t byte = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          byte = 2 * byte + (to_f32(v[i][e]) + off[e] > 0.0f ? 1u : 0u);
        const uint32_t word = or_quad(byte << (24 - 8 * (lane & 3)));
        if ((lane & 3) == 0 && k < a.K) bits[static_cast<size_t>(p) * kw + k / 32] = word;
      }
    }
    return;
  }
  const int l = lora_adapter(a, row);
  if (l < 0) return;
  const T* w = static_cast<const T*>(a.a) + (static_cast<size_t>(l) * a.rank + r) * a.K;
  float sum = 0.0f;
  for (int k0 = 0; k0 < a.K; k0 += 512 * kAhead) {
    T xv[kAhead][8], wv[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = k0 + 512 * i + 8 * lane;
      if (k0 + 512 * i < a.K) {
        load8(xv[i], x + k, a.K - k);
        load8(wv[i], w + k, a.K - k);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k0 + 512 * i >= a.K) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += to_f32(xv[i][e]) * to_f32(wv[i][e]);
    }
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
  if (lane == 0) u[static_cast<size_t>(p) * a.rank + r] = sum * (a.scale ? a.scale[l] : 1.0f);
}

// --------------------------------------------------------- bits, u -> y ---
struct UsArgs {
  LoraArgs a;
  const float* u;  // [slices][M][rank]
  const uint32_t* bits;
  uint32_t bits_bytes, w_bytes, tmask;
  int32_t Kw, chunks, Nw, slices;
};

template <class T, class Y, int NW>
__global__ __launch_bounds__(64 * NW) void lora_up_skinny_kernel(UsArgs g) {
  constexpr int kPart = (NW - 1) * 64 * kSkinnyStride;
  __shared__ __attribute__((aligned(16))) float part[kPart], low_part[kPart];
  const LoraArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, c = lane & 31;
  const int rt = blockIdx.x / g.Nw, n0 = 32 * (blockIdx.x - rt * g.Nw);
  const int p = 32 * rt + c;
  SkinnyTile t;
  t.ra = tile_rsrc(g.bits, g.bits_bytes);
  t.rb = tile_rsrc(a.w, g.w_bytes);
  t.aoff = static_cast<uint32_t>(min(p, a.M - 1)) * g.Kw * 4 + 16 * h;
  t.boff = static_cast<uint32_t>(n0 + c) * g.Kw * 4 + 16 * h;
  t.K = a.K;
  t.Kw = g.Kw;
  t.chunks = g.chunks;
  t.tmask = g.tmask;
  const int row = lora_row(a, p);
  const int id = p < a.M ? lora_adapter(a, row) : -1;
  // u b^T: 16 ranks of an adapter are a job of wave (adapter + ranks / 16) mod
  // NW, so that a row's sums do not hang on which rows lie beside it.  The first
  // jobs' values are loaded before the binary products.
  const uint32_t have = static_cast<uint32_t>(__ballot(id >= 0));
  float v[8];            // u, 16 ranks of the row
  int l[kAdapters];
  RawB<T> b[kAdapters];  // and of this output's rows of b
  auto load_u = [&](int r) {
    const int rr = r + 8 * h;
    const float* src =
        g.u + (id >= 0 && rr < a.rank ? static_cast<size_t>(p) * a.rank + rr : size_t{0});
    __builtin_memcpy(v, __builtin_assume_aligned(src, 16), sizeof(v));
    for (int s = 1; s < g.slices; ++s) {
      float w[8];
      __builtin_memcpy(
          w, __builtin_assume_aligned(src + static_cast<size_t>(s) * a.M * a.rank, 16), sizeof(w));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
  };
  // This wave's next adapters among `todo` for ranks r .., their rows of b.
  auto load_adapters = [&](uint32_t& todo, int r) {
#pragma unroll
    for (int i = 0; i < kAdapters; ++i) {
      l[i] = -1;
      while (todo && l[i] < 0) {
        const int q = __builtin_amdgcn_readlane(id, __builtin_ctz(todo));
        todo &= ~static_cast<uint32_t>(__ballot(id == q));
        if (((q + (r >> 4)) & (NW - 1)) == wave) l[i] = q;
      }
      if (l[i] >= 0) b[i] = load_b<T>(a, l[i], n0 + c, r + 8 * h);
    }
  };
  uint32_t todo = have;
  if (have) {
    load_u(0);
    load_adapters(todo, 0);
  }
  v16f acc = skinny_part<NW>(t, wave, h);
  v16f low = {};
  for (int r = 0; have && r < a.rank;) {
    const bool in = r + 8 * h < a.rank;
    v8bf uf[3];
    split_frag<3>(v, in, uf);
#pragma unroll
    for (int i = 0; i < kAdapters; ++i) {
      if (l[i] < 0) continue;
      v8bf bf[kParts<T>];
      split_b<T>(b[i], in && n0 + c < a.N, bf);
      add_rows<T>(low, bf, uf, id == l[i]);
    }
    if (!todo) {
      r += 16;
      if (r >= a.rank) break;
      todo = have;
      load_u(r);
    }
    load_adapters(todo, r);
  }
  skinny_join<NW>(acc, part, wave, lane);
  if (have) skinny_join<NW>(low, low_part, wave, lane);
  if (wave > 0 || p >= a.M) return;
  const __amdgpu_buffer_rsrc_t ral = tile_rsrc(a.alpha, a.alpha ? a.N * 4 : 0);
  Y* dst = static_cast<Y*>(a.y) + static_cast<size_t>(row) * a.N + n0;
#pragma unroll
  for (int e = 0; e < 16; e += 4) {
    // Registers e .. e + 3 hold four consecutive outputs of row c.
    const int n = 2 * e + 4 * h;
    const v4i f = tile_load4(ral, (n0 + n) * 4, 0);
    Y y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y[i] = from_f32<Y>(acc[e + i] * (a.alpha ? __int_as_float(f[i]) : 1.0f) + low[e + i]);
    if (n0 + n + 4 <= a.N) {
      __builtin_memcpy(dst + n, y, sizeof(y));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + n + i < a.N) dst[n + i] = y[i];
    }
  }
}

}  // namespace

void launch_lora_down_rows(const LoraArgs& a, float* u, uint32_t* bits, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(a.M), static_cast<unsigned>((a.rank + kNW) / kNW));
  with_real_type(a.dtype, [&](auto v) {
    lora_down_rows_kernel<decltype(v)><<<grid, kNT, 0, s>>>(a, u, bits);
  });
}

void launch_lora_up_skinny(const LoraArgs& a, const float* u, const uint32_t* bits, int slices,
                           hipStream_t s) {
  UsArgs g;
  g.a = a;
  g.u = u;
  g.bits = bits;
  g.slices = slices;
  g.Kw = static_cast<int32_t>(words_of(a.K));
  g.bits_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.M) * g.Kw * 4);
  g.w_bytes = static_cast<uint32_t>(static_cast<int64_t>(a.N) * g.Kw * 4);
  g.tmask = tail_mask(a.K);
  g.chunks = (g.Kw + 7) / 8;
  g.Nw = static_cast<int32_t>(words_of(a.N));
  const unsigned grid = static_cast<unsigned>((a.M + 31) / 32 * g.Nw);
  with_real_type(a.dtype, [&](auto v) {
    using T = decltype(v);
    with_real_type(a.out_dtype, [&](auto y) {
      using Y = decltype(y);
      switch (skinny_waves(g.chunks)) {
        case 8: lora_up_skinny_kernel<T, Y, 8><<<grid, 64 * 8, 0, s>>>(g); break;
        case 4: lora_up_skinny_kernel<T, Y, 4><<<grid, 64 * 4, 0, s>>>(g); break;
        default: lora_up_skinny_kernel<T, Y, 2><<<grid, 64 * 2, 0, s>>>(g); break;
      }
    });
  });
}

}  // namespace bnn
