// Root-mean-square norm with the residual's addition and an output in 8 bits
// (bnn_rmsnorm).  One pass: a row stays in the registers of its W waves, 8
// values at a time per lane, from the sum of squares and the largest |h w| to
// the rounding.  Bound by memory: 8192 x 4096 bf16 with a residual in 42-50 us
// from card to card (45.8: 5.1 TB/s, a large copy's rate), fp32 in 84-88 us, 5.0
// to 5.2 TB/s.  16-bit rows under fp32 weights go in 64 bits throughout and are
// bound by those: 59-62 us, 3.8 to 4.0 TB/s.
//
// r cancels in q = rint(127 p / max p), p = h w, which is rounded as if from the
// exact p: where the quotient comes near a border n + 1/2 (within 2^-13, many
// times its error of at most 127 * 3 * 2^-24), it is divided again in 64 bits;
// else it is rounded as it is.
//
// Rows and weights of 16 bits: p is exact in fp32 (8 + 8 or 11 + 11 bits), and so
// is its largest; sums and quotients are fp32's, as long as the largest p, the
// sum of squares and eps lie well inside its range (only p's that are 2^43 times
// smaller than the largest may lie below it, and y lose bits there).  Other rows
// (infinities, NaN and rows of zeros among them), and rows or weights of fp32, go
// in 64 bits.
#include "dtypes.hpp"
#include "quant.hpp"
#include "wave_ops.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;

struct NormRow {
  double ss;   // sum of h^2
  double top;  // max |h w|
};

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// 8 values of a row, wherever it lies: whole 16-byte accesses, aligned to the
// element only.
template <class T>
struct Eight {
  T v[8];
};

template <class T>
__device__ __forceinline__ Eight<T> load8(const T* p, int n) {
  Eight<T> e;
  if (n >= 8) {
    constexpr int kParts = sizeof(T) / 2;
    u32x4_any raw[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) raw[i] = reinterpret_cast<const u32x4_any*>(p)[i];
    __builtin_memcpy(&e, raw, sizeof(e));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = i < n ? p[i] : T(0.0f);
  }
  return e;
}

template <class T>
__device__ __forceinline__ void store8(T* p, const Eight<T>& e, int n) {
  if (n >= 8) {
    constexpr int kParts = sizeof(T) / 2;
    u32x4_any raw[kParts];
    __builtin_memcpy(raw, &e, sizeof(e));
#pragma unroll
    for (int i = 0; i < kParts; ++i) reinterpret_cast<u32x4_any*>(p)[i] = raw[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = e.v[i];
  }
}

// 8 of a row's bytes, n of them in the row.
__device__ __forceinline__ void store_q(int8_t* q, uint32_t b0, uint32_t b1, int n) {
  if (n >= 8) {
    *reinterpret_cast<u32x2_any*>(q) = u32x2_any{b0, b1};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) q[i] = static_cast<int8_t>((i < 4 ? b0 : b1) >> (8 * (i % 4)));
  }
}

// The fp32 totals of a row over its W waves.
template <int W>
__device__ __forceinline__ void row_totals(float& ss, float& top, float (*part)[2]) {
  ss = wave_sum(ss);
  top = wave_max(top);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      part[wave][0] = ss;
      part[wave][1] = top;
    }
    __syncthreads();
    ss = part[0][0];
    top = part[0][1];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      ss += part[w][0];
      top = __builtin_fmaxf(top, part[w][1]);
    }
  }
}

// The row's totals over its W waves (in a workgroup of 4 / W rows, or of W waves).
template <int W>
__device__ __forceinline__ NormRow row_totals(NormRow r, double (*part)[2]) {
  r.ss = wave_sum(r.ss);
  r.top = wave_max(r.top);
  if constexpr (W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      part[wave][0] = r.ss;
      part[wave][1] = r.top;
    }
    __syncthreads();
    r.ss = part[0][0];
    r.top = part[0][1];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      r.ss += part[w][0];
      r.top = fmax(r.top, part[w][1]);
    }
  }
  return r;
}

// A row per W waves; a lane holds up to G groups of 8 values.
template <class T, class TW, int W, int G>
__global__ __launch_bounds__(W > 4 ? W * 64 : kNT) void rmsnorm_kernel(NormArgs a) {
  __shared__ double part[W][2];
  constexpr int kRows = W > 4 ? 1 : 4 / W;
  const int lane = threadIdx.x % (W * 64);
  const int64_t m = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / (W * 64);
  if (m >= a.M) return;  // (a row's whole waves; with W > 1 the workgroup has one row)
  static_assert(W == 1 || W >= 4, "rows that share a workgroup need no barrier");
  const T* x = static_cast<const T*>(a.x) + m * a.x_stride;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + m * a.r_stride : nullptr;
  const TW* weight = static_cast<const TW*>(a.weight);
  const int D = a.D;

  auto weight8 = [&](int d) {
    Eight<TW> w;
    if (weight) return load8(weight + d, D - d);
#pragma unroll
    for (int i = 0; i < 8; ++i) w.v[i] = TW(1.0f);
    return w;
  };
  constexpr bool kNarrow = sizeof(T) == 2 && sizeof(TW) == 2;
  Eight<TW> held[kNarrow ? G : 1];  // (asked for with the rows: their wait is one)

  Eight<T> h[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int d = 8 * (lane + g * W * 64);
    if (d < D) h[g] = load8(x + d, D - d);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) h[g].v[i] = T(0.0f);
  }
  auto hold_weight = [&]() {
    if constexpr (kNarrow) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int d = 8 * (lane + g * W * 64);
        held[g] = d < D ? weight8(d) : Eight<TW>{};
      }
    }
  };
  if (res) {
    Eight<T> r[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int d = 8 * (lane + g * W * 64);
      r[g] = d < D ? load8(res + d, D - d) : Eight<T>{};
    }
    hold_weight();
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[g].v[i] = from_f32<T>(to_f32(h[g].v[i]) + to_f32(r[g].v[i]));
  } else {
    hold_weight();
  }
  if (a.sum) {
    T* sum = static_cast<T*>(a.sum) + m * D;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int d = 8 * (lane + g * W * 64);
      if (d < D) store8(sum + d, h[g], D - d);
    }
  }
  if constexpr (kNarrow) {
    __shared__ float totals[W][2];
    float p[G][8], ss = 0.0f, top = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const Eight<TW>& w = held[g];
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = to_f32(h[g].v[i]);
        sq = __builtin_fmaf(v, v, sq);
        p[g][i] = v * to_f32(w.v[i]);
        top = __builtin_fmaxf(top, __builtin_fabsf(p[g][i]));
      }
      ss += sq;
    }
    row_totals<W>(ss, top, totals);
    const float mean = ss / static_cast<float>(D) + a.eps;
    if (ss > 1e-25f && ss < 1e37f && mean < 1e37f && top > 1e-25f && top < 1e37f) {
      const float rstd = 1.0f / __builtin_sqrtf(mean);
      // (the largest |y| may lie beyond fp32 where its 127th part does not)
      const float most = top * rstd;
      if (a.q && lane == 0) a.scale[m] = most < __builtin_inff() ? most / 127.0f : top / 127.0f * rstd;
      const float inv = 127.0f / top;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int d = 8 * (lane + g * W * 64);
        if (d >= D) break;
        if (a.y) {
          Eight<T> y;
#pragma unroll
          for (int i = 0; i < 8; ++i) y.v[i] = from_f32<T>(p[g][i] * rstd);
          store8(static_cast<T*>(a.y) + m * D + d, y, D - d);
        }
        if (a.q) {
          // 1.5 * 2^23 added: fp32 rounds to whole numbers there, and its low
          // byte is that number's
          constexpr float kWhole = 12582912.0f;
          float t[8], near = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            t[i] = __builtin_fmaf(p[g][i], inv, kWhole);
            near = __builtin_fmaxf(near, __builtin_fabsf(__builtin_fmaf(p[g][i], inv, kWhole - t[i])));
          }
          if (near > 0.5f - 0x1p-13f) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              t[i] = kWhole + static_cast<float>(__builtin_rint(127.0 * static_cast<double>(p[g][i]) /
                                                                static_cast<double>(top)));
          }
          auto bits = [&](int i) { return __builtin_bit_cast(uint32_t, t[i]); };
          // (v_perm: bytes 0-3 of its second operand, 4-7 of its first)
          auto four = [&](int i) {
            return __builtin_amdgcn_perm(__builtin_amdgcn_perm(bits(i + 3), bits(i + 2), 0x0c0c0400),
                                         __builtin_amdgcn_perm(bits(i + 1), bits(i), 0x0c0c0400), 0x05040100);
          };
          store_q(a.q + m * a.q_stride + d, four(0), four(4), D - d);
        }
      }
      return;
    }
  }

  NormRow r = {0.0, 0.0};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int d = 8 * (lane + g * W * 64);
    if (d >= D) break;
    const Eight<TW> w = weight8(d);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double v = to_f32(h[g].v[i]);
      r.ss = __builtin_fma(v, v, r.ss);
      r.top = fmax(r.top, __builtin_fabs(v * static_cast<double>(to_f32(w.v[i]))));
    }
  }
  r = row_totals<W>(r, part);
  const bool bad = !(r.ss < __builtin_inf());
  const double root = __builtin_sqrt(r.ss / D + static_cast<double>(a.eps));
  const double rstd = bad ? __builtin_nan("") : root > 0.0 ? 1.0 / root : 0.0;
  if (a.q && lane == 0) a.scale[m] = static_cast<float>(r.top * rstd / 127.0);
  const double inv = bad || !(r.top > 0.0) ? 0.0 : 127.0 / r.top;

#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int d = 8 * (lane + g * W * 64);
    if (d >= D) break;
    const Eight<TW> w = weight8(d);
    double p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      p[i] = static_cast<double>(to_f32(h[g].v[i])) * static_cast<double>(to_f32(w.v[i]));
    if (a.y) {
      Eight<T> y;
#pragma unroll
      for (int i = 0; i < 8; ++i) y.v[i] = from_f32<T>(static_cast<float>(p[i] * rstd));
      store8(static_cast<T*>(a.y) + m * D + d, y, D - d);
    }
    if (a.q) {
      float t[8];
      float near = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = bad ? 0.0f : static_cast<float>(p[i] * inv);
        t[i] = __builtin_rintf(f);
        near = fmaxf(near, __builtin_fabsf(f - t[i]));
      }
      if (near > 0.5f - 0x1p-13f) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (inv > 0.0) t[i] = static_cast<float>(__builtin_rint(127.0 * p[i] / r.top));
      }
      uint32_t b[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        b[i / 4] |= (static_cast<uint32_t>(static_cast<int>(t[i])) & 0xFFu) << (8 * (i % 4));
      store_q(a.q + m * a.q_stride + d, b[0], b[1], D - d);
    }
  }
}

template <class T, class TW>
void launch_types(const NormArgs& a, hipStream_t s) {
  auto go = [&](auto wc, auto gc) {
    constexpr int W = decltype(wc)::value, G = decltype(gc)::value;
    constexpr int kRows = W > 4 ? 1 : 4 / W;
    // (a launch's work-items stay below 2^32: 2^21 workgroups of up to 1024)
    constexpr int64_t kMost = int64_t{kRows} << 21;
    for (int64_t m = 0; m < a.M; m += kMost) {
      NormArgs b = a;
      b.M = a.M - m < kMost ? a.M - m : kMost;
      auto at = [&](const void* p, int64_t stride, size_t size) -> const void* {
        return p ? static_cast<const char*>(p) + m * stride * static_cast<int64_t>(size) : nullptr;
      };
      b.x = at(a.x, a.x_stride, sizeof(T));
      b.residual = at(a.residual, a.r_stride, sizeof(T));
      b.sum = const_cast<void*>(at(a.sum, a.D, sizeof(T)));
      b.y = const_cast<void*>(at(a.y, a.D, sizeof(T)));
      b.q = a.q ? a.q + m * a.q_stride : nullptr;
      b.scale = a.q ? a.scale + m : nullptr;
      const unsigned grid = static_cast<unsigned>((b.M + kRows - 1) / kRows);
      rmsnorm_kernel<T, TW, W, G><<<grid, W > 4 ? W * 64 : kNT, 0, s>>>(b);
    }
  };
  const int groups = (a.D + 7) / 8;
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  using Two = integral_constant<int, 2>;
  using Four = integral_constant<int, 4>;
  using Eight_ = integral_constant<int, 8>;
  // Where there are rows for all CUs, rows up to 1536 values go to a wave each
  // (us, bf16 with residual, one wave : four waves: 32768 x 1024 47 : 57, 32768 x
  // 600 36 : 52; 16384 x 1100 fp32 32 : 40; 16384 x 2048 50 : 45); a few rows are
  // done sooner by four (301 x 1024 4.8 : 4.0).  Longer rows, eight waves : four :
  // sixteen: 8192 x 4096 45.8 : 46.5 : 86; eight : sixteen: 4096 x 8192 48 : 65,
  // 2048 x 16384 54 : 60.
  const bool many = a.M >= 4096;
  if (groups <= 64) return go(One{}, One{});
  if (many && groups <= 128) return go(One{}, Two{});
  if (many && groups <= 192) return go(One{}, Four{});
  if (groups <= 256) return go(Four{}, One{});
  if (groups <= 512) return go(Eight_{}, One{});
  if (groups <= 1024) return go(Eight_{}, Two{});
  if (groups <= 2048) return go(Eight_{}, Four{});
  return go(integral_constant<int, 16>{}, Eight_{});
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s) {
  with_real_type(a.dtype, [&](auto t) {
    using T = decltype(t);
    if (a.weight_dtype == BNN_F32) launch_types<T, float>(a, s);
    else launch_types<T, T>(a, s);
  });
  return hipGetLastError();
}

}  // namespace bnn
