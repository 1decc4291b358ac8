// Root-mean-square norm with the residual's addition and an output in 8 bits
// (bnn_rmsnorm).  One pass: a row stays in the registers of its W waves, 8
// values at a time per lane, from the sum of squares and the largest |h w| to
// the rounding.
//
// r cancels in q = rint(127 p / max p), p = h w.  Where both are 16-bit values
// p is exact in fp32, and the quotient of the 23-bit 127 p by max p comes no
// nearer to a border n + 1/2 than 2^-24 of it without lying on it; products of
// fp32 values need 64 bits.  So a value whose fp32 quotient comes near a border
// (within 2^-13, far more than its error) is divided again in 64 bits; the rest
// is rounded as it is.
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

  Eight<T> h[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const int d = 8 * (lane + g * W * 64);
    if (d < D) h[g] = load8(x + d, D - d);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) h[g].v[i] = T(0.0f);
  }
  if (res) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int d = 8 * (lane + g * W * 64);
      if (d >= D) break;
      const Eight<T> r = load8(res + d, D - d);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[g].v[i] = from_f32<T>(to_f32(h[g].v[i]) + to_f32(r.v[i]));
    }
  }
  if (a.sum) {
    T* sum = static_cast<T*>(a.sum) + m * D;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int d = 8 * (lane + g * W * 64);
      if (d < D) store8(sum + d, h[g], D - d);
    }
  }
  auto weight8 = [&](int d) {
    Eight<TW> w;
    if (weight) return load8(weight + d, D - d);
#pragma unroll
    for (int i = 0; i < 8; ++i) w.v[i] = TW(1.0f);
    return w;
  };

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
      int8_t* q = a.q + m * a.q_stride + d;
      if (D - d >= 8) {
        *reinterpret_cast<u32x2_any*>(q) = u32x2_any{b[0], b[1]};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < D - d) q[i] = static_cast<int8_t>(b[i / 4] >> (8 * (i % 4)));
      }
    }
  }
}

template <class T, class TW>
void launch_types(const NormArgs& a, hipStream_t s) {
  auto go = [&](auto wc, auto gc) {
    constexpr int W = decltype(wc)::value, G = decltype(gc)::value;
    constexpr int kRows = W > 4 ? 1 : 4 / W;
    const unsigned grid = static_cast<unsigned>((a.M + kRows - 1) / kRows);
    rmsnorm_kernel<T, TW, W, G><<<grid, W > 4 ? W * 64 : kNT, 0, s>>>(a);
  };
  const int groups = (a.D + 7) / 8;
#ifdef NORM_FORCE
  return go(std::integral_constant<int, NORM_W>{}, std::integral_constant<int, NORM_G>{});
#endif
  using std::integral_constant;
  if (groups <= 64) return go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  if (groups <= 256) return go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  if (groups <= 512) return go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  if (groups <= 1024) return go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  if (groups <= 2048) return go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 16>{}, integral_constant<int, 8>{});
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
