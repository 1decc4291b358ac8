// Log probabilities of given answers, the entropy and the largest alternatives
// of a row of logits (bnn_logprobs), in one pass over them.
//
// Sums, per wave, in units of log2 with c = logit_scale * log2(e):
//   s1 = sum 2^d,  s2 = sum 2^d d,   d = c v - ref,
//   ln p_v = (c v - ref - log2 s1) ln 2,   entropy = (log2 s1 - s2 / s1) ln 2.
// ref is any number near the largest c v: it is taken from the first values and
// moved (s1 and s2 with it) only when a value lies 2^60 above it, so that a
// value costs one fma, one exp2 and two sums, and no maximum of its own.
//
// The alternatives so far are a sorted list over the wave's lanes, one 64-bit
// key each: the value's order in the high word, the inverted index in the low
// one.  A group of 8 values per lane is looked at further only where its largest
// reaches the top_k-th key, and values are inserted one by one; where many do
// (the first group, rising rows), the bound is first raised to what top_k lanes'
// largest values reach.
#include "dtypes.hpp"
#include "quant.hpp"

#include <type_traits>

namespace bnn {
namespace {

constexpr int kNT = 256;
constexpr int kGroup = 512;   // values of a wave's step: 8 per lane
constexpr float kAway = 60.0f;
constexpr float kFar = 3e38f;

struct Sums {
  double ref;
  float s1, s2;
};

struct alignas(16) Part {  // followed by top_k keys
  Sums sums;
};
__host__ __device__ inline size_t part_bytes(int top_k) {
  return (sizeof(Part) + size_t{8} * top_k + 15) / 16 * 16;
}

template <class T> struct RawOf { using type = float; };
template <> struct RawOf<int32_t> { using type = int32_t; };

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The order of values as unsigned integers; kFloor lies above -inf's.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);  // (-0 is 0)
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t order_of(int32_t v) {
  return static_cast<uint32_t>(v) ^ 0x80000000u;
}
__device__ __forceinline__ void value_of(uint32_t o, float& v) {
  v = __builtin_bit_cast(float, o ^ (o & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ void value_of(uint32_t o, int32_t& v) {
  v = static_cast<int32_t>(o ^ 0x80000000u);
}
template <class R>
constexpr uint32_t kFloor = std::is_same<R, float>::value ? 0x00800000u : 0u;

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// 8 values from p on, aligned to their element only.
template <class T>
struct Eight {
  T v[8];
};
template <class T>
__device__ __forceinline__ Eight<T> load8(const T* p) {
  Eight<T> e;
  constexpr int kParts = sizeof(T) / 2;
  u32x4_any raw[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) raw[i] = reinterpret_cast<const u32x4_any*>(p)[i];
  __builtin_memcpy(&e, raw, sizeof(e));
  return e;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v = __builtin_fmaxf(v, __shfl_xor(v, o));
  return v;
}

// A wave's sorted list of keys, the largest in lane 0; bound is the key of lane
// top_k - 1 (0: the list is not full), floor what a value's order must reach.
struct Top {
  uint32_t hi, lo;  // this lane's key
  uint32_t floor;   // uniform
  uint64_t bound;   // uniform

  __device__ __forceinline__ void insert(uint64_t key, int top_k) {
    const uint64_t mine = static_cast<uint64_t>(hi) << 32 | lo;
    const int pos = __popcll(__ballot(mine > key));
    const int lane = threadIdx.x & 63;
    const uint32_t uh = __shfl_up(hi, 1), ul = __shfl_up(lo, 1);
    hi = lane < pos ? hi : lane == pos ? static_cast<uint32_t>(key >> 32) : uh;
    lo = lane < pos ? lo : lane == pos ? static_cast<uint32_t>(key) : ul;
    const uint32_t bh = __builtin_amdgcn_readlane(hi, top_k - 1);
    bound = static_cast<uint64_t>(bh) << 32 |
            static_cast<uint32_t>(__builtin_amdgcn_readlane(lo, top_k - 1));
    if (bh > floor) floor = bh;
  }
};

// Raises top.floor to an order that the values of at least top_k lanes reach, if
// there is a higher one (to 16 bits: a lower bound is all it is).
__device__ __forceinline__ void raise_floor(Top& top, uint32_t mine, int top_k) {
  uint32_t at = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t next = at | 1u << b;
    if (__popcll(__ballot(mine >= next)) >= top_k) at = next;
  }
  if (at > top.floor) top.floor = at;
}

// SAFE: the reference is the largest value itself and differences are taken
// before the factor, for rows whose c v leave fp32's range, rows without a value
// in reach and rows with NaN or infinity.
template <bool SAFE>
struct Scan {
  float c, ref, s1, s2;

  __device__ __forceinline__ void start(float factor) {
    c = factor;
    ref = SAFE ? -__builtin_inff() : -kFar;
    s1 = s2 = 0.0f;
  }
  __device__ __forceinline__ float delta(float v) const {
    if constexpr (SAFE) return v == -__builtin_inff() ? v : (v - ref) * c;
    else return __builtin_fmaf(v, c, -ref);
  }
  __device__ __forceinline__ void add(const float (&v)[8], float fm) {
    if (__any(SAFE ? fm > ref : delta(fm) > kAway)) {
      const float top = wave_max(fm);
      const float next = SAFE ? top : __builtin_fminf(__builtin_fmaxf(top * c, -kFar), kFar);
      float move = SAFE ? (ref - next) * c : ref - next;
      move = s1 > 0.0f ? __builtin_fmaxf(move, -1e4f) : -1e4f;
      const float f = exp2_of(move);
      s2 = f * __builtin_fmaf(move, s1, s2);
      s1 *= f;
      ref = next;
    }
    float e[8], d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      d[i] = delta(v[i]);
      e[i] = exp2_of(d[i]);
      d[i] = __builtin_fmaxf(d[i], -200.0f);  // (0 * -inf)
    }
    s1 += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    float t = e[0] * d[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = __builtin_fmaf(e[i], d[i], t);
    s2 += t;
  }
  __device__ __forceinline__ Sums total() const {
    return {SAFE ? static_cast<double>(ref) * c : static_cast<double>(ref), wave_sum(s1),
            wave_sum(s2)};
  }
};

// Sums over both sets of values.  (A set without a value in reach: s1 0.)
__device__ __forceinline__ Sums joined(const Sums& a, const Sums& b) {
  if (b.s1 == 0.0f) return a;
  if (a.s1 == 0.0f) return b;
  const double ref = fmax(a.ref, b.ref);
  const float ma = fmaxf(static_cast<float>(a.ref - ref), -1e4f);
  const float mb = fmaxf(static_cast<float>(b.ref - ref), -1e4f);
  const float fa = exp2_of(ma), fb = exp2_of(mb);
  return {ref, fa * a.s1 + fb * b.s1,
          fa * __builtin_fmaf(ma, a.s1, a.s2) + fb * __builtin_fmaf(mb, b.s1, b.s2)};
}

// Values [begin, end) of a row, by wave `wave` of `waves`.
template <class T, bool SAFE, bool TOP>
__device__ __forceinline__ Sums scan(const T* row, int begin, int end, int wave, int waves,
                                     float c, int top_k, Top& top) {
  using R = typename RawOf<T>::type;
  constexpr bool kInts = std::is_same<R, int32_t>::value;
  const int lane = threadIdx.x & 63;
  Scan<SAFE> sc;
  sc.start(c);
  // 8 values per lane from index `at` on, the lane's first n of them in the row.
  auto step = [&](const R (&v)[8], int at, int n, auto part) {
    constexpr bool kPart = decltype(part)::value;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f[i] = !kPart || i < n ? static_cast<float>(v[i]) : -__builtin_inff();
    float most = f[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most = __builtin_fmaxf(most, f[i]);
    sc.add(f, most);
    if constexpr (TOP) {
      uint32_t mo;
      if constexpr (kInts) {  // (beyond 2^24 their order is not that of f)
        R m = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i)
          if (!kPart || i < n) m = m > v[i] ? m : v[i];
        mo = kPart && n <= 0 ? 0u : order_of(m);
      } else {
        mo = order_of(most);
      }
      const uint64_t reach = __ballot(mo >= top.floor);
      if (reach) {
        if (__popcll(reach) > 12) raise_floor(top, mo, top_k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t o = order_of(v[i]);
          uint64_t mask = __ballot(o >= top.floor && (!kPart || i < n));
          while (mask) {
            const int l = __builtin_ctzll(mask);
            mask &= mask - 1;
            const uint32_t oh = __builtin_amdgcn_readlane(o, l);
            const uint32_t index = static_cast<uint32_t>(at + 8 * l + i);
            const uint64_t key = static_cast<uint64_t>(oh) << 32 | static_cast<uint32_t>(~index);
            if (key > top.bound) top.insert(key, top_k);
          }
        }
      }
    }
  };
  for (int at = begin + wave * kGroup; at < end; at += waves * kGroup) {
    const int i0 = at + 8 * lane;
    R v[8];
    if (at + kGroup <= end) {
      const Eight<T> e = load8(row + i0);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = static_cast<R>(e.v[i]);
      step(v, at, 8, std::false_type{});
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i0 + i < end ? static_cast<R>(row[i0 + i]) : R(0);
      step(v, at, end - i0, std::true_type{});
    }
  }
  return sc.total();
}

// A wave's sums: in fp32's range by the quick form, or else by the safe one.
template <class T, bool TOP>
__device__ __forceinline__ Sums wave_part(const T* row, int begin, int end, int wave, int waves,
                                          float c, int top_k, Top& top) {
  Sums s = scan<T, false, TOP>(row, begin, end, wave, waves, c, top_k, top);
  if (!(s.s1 > 0.0f && s.s1 < __builtin_inff()))
    s = scan<T, true, false>(row, begin, end, wave, waves, c, top_k, top);
  return s;
}

// A row's outputs from its sums and (lane j: the j-th) keys, by one wave.
template <class T>
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int64_t t, const Sums& s,
                                          uint64_t key, float c) {
  using R = typename RawOf<T>::type;
  constexpr double kLn2 = 0.693147180559945309417;
  const int lane = threadIdx.x & 63;
  const bool none = s.s1 == 0.0f, bad = !(s.s1 < __builtin_inff());
  const float ls = log2f(s.s1);
  const float nan = __builtin_nanf("");
  auto ln_p = [&](R v) {
    if (std::is_same<R, float>::value && static_cast<float>(v) == -__builtin_inff())
      return -__builtin_inff();
    return static_cast<float>((static_cast<double>(v) * c - s.ref - static_cast<double>(ls)) * kLn2);
  };
  if (a.entropy && lane == 0)
    a.entropy[t] = bad ? nan : none ? 0.0f
        : static_cast<float>(static_cast<double>(ls - s.s2 / s.s1) * kLn2);
  for (int j = lane; j < a.n; j += 64) {
    const int id = a.ids[t * a.n + j];
    float lp = -__builtin_inff();
    if (id >= 0 && id < a.V) {
      const R v = static_cast<R>(static_cast<const T*>(a.logits)[t * a.stride + id]);
      if (bad) lp = nan;
      else if (!none) lp = ln_p(v);
    }
    a.logp[t * a.n + j] = lp;
  }
  if (lane < a.top_k) {
    const bool is = key != 0 && !bad && !none;
    R v;
    value_of(static_cast<uint32_t>(key >> 32), v);
    a.top_ids[t * a.top_k + lane] = is ? static_cast<int32_t>(~static_cast<uint32_t>(key)) : -1;
    a.top_logp[t * a.top_k + lane] = bad ? nan : is ? ln_p(v) : -__builtin_inff();
  }
}

__device__ __forceinline__ float factor_of(float scale) {
  return static_cast<float>(static_cast<double>(scale) * 1.44269504088896340736);
}

// W waves per part of a row: whole rows (splits 1), or parts to the workspace.
template <class T, int W, bool TOP>
__global__ __launch_bounds__(kNT) void logprobs_kernel(LogprobsArgs a, int splits, int length) {
  using R = typename RawOf<T>::type;
  __shared__ Sums sums[W];
  __shared__ uint64_t keys[W][BNN_MAX_ALTERNATIVES];
  constexpr int kParts = kNT / 64 / W;  // of a workgroup
  const int lane = threadIdx.x & 63;
  const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t part = static_cast<int64_t>(blockIdx.x) * kParts +
                       (W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  const int64_t t = part / splits;
  if (t >= a.T) return;
  const int begin = static_cast<int>(part % splits) * length;
  const int end = min(begin + length, a.V);
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float c = factor_of(a.scale);
  Top top = {0, 0, kFloor<R>, 0};
  Sums s = wave_part<T, TOP>(row, begin, end, wave, W, c, a.top_k, top);
  if constexpr (W > 1) {
    if (lane == 0) sums[wave] = s;
    if (TOP && lane < a.top_k)
      keys[wave][lane] = static_cast<uint64_t>(top.hi) << 32 | top.lo;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll 1
    for (int w = 1; w < W; ++w) {
      s = joined(s, sums[w]);
      if constexpr (TOP) {
        for (int j = 0; j < a.top_k; ++j) {
          const uint64_t key = keys[w][j];
          if (!(key > top.bound)) break;
          top.insert(key, a.top_k);
        }
      }
    }
  }
  const uint64_t key = static_cast<uint64_t>(top.hi) << 32 | top.lo;
  if (splits == 1) {
    write_row<T>(a, t, s, key, c);
  } else {
    char* out = static_cast<char*>(a.workspace) + part * part_bytes(a.top_k);
    if (lane == 0) reinterpret_cast<Part*>(out)->sums = s;
    if (TOP && lane < a.top_k) reinterpret_cast<uint64_t*>(out + sizeof(Part))[lane] = key;
  }
}

// A row's parts put together, by one wave.
template <class T>
__global__ __launch_bounds__(64) void join_kernel(LogprobsArgs a, int splits) {
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x;
  const char* at = static_cast<const char*>(a.workspace) + t * splits * part_bytes(a.top_k);
  Sums s = {0.0, 0.0f, 0.0f};
  Top top = {0, 0, 0, 0};
  for (int p = 0; p < splits; ++p) {
    const char* part = at + p * part_bytes(a.top_k);
    s = joined(s, reinterpret_cast<const Part*>(part)->sums);
    for (int j = 0; j < a.top_k; ++j) {
      const uint64_t key = reinterpret_cast<const uint64_t*>(part + sizeof(Part))[j];
      if (!(key > top.bound)) break;
      top.insert(key, a.top_k);
    }
  }
  (void)lane;
  write_row<T>(a, t, s, static_cast<uint64_t>(top.hi) << 32 | top.lo, factor_of(a.scale));
}

constexpr int kParts = 1024;     // parts that fill the card
constexpr int kLength = 2048;    // a part's values, at least

int64_t most_splits(int32_t V) { return (V + kLength - 1) / kLength; }
int64_t splits_of(int64_t T, int32_t V) {
  const int64_t want = (kParts + T - 1) / T;
  return want < most_splits(V) ? want : most_splits(V);
}

}  // namespace

// (Rows times splits never pass kParts + T - 1 with T < kParts, nor T times the
// most splits: a bound that does not fall as T grows.)
size_t logprobs_workspace(int64_t T, int32_t V, int32_t top_k) {
  if (most_splits(V) < 2) return 0;
  const int64_t parts = T * most_splits(V) < 2 * kParts ? T * most_splits(V) : 2 * kParts;
  return static_cast<size_t>(parts) * part_bytes(top_k);
}

hipError_t launch_logprobs(const LogprobsArgs& a, hipStream_t s) {
  const int splits = static_cast<int>(splits_of(a.T, a.V));
  const int length = ((a.V + splits - 1) / splits + kGroup - 1) / kGroup * kGroup;
  auto go = [&](auto t) {
    using T = decltype(t);
    auto with = [&](auto wc, auto tc) {
      constexpr int W = decltype(wc)::value;
      constexpr int per = kNT / 64 / W;
      const int64_t parts = a.T * splits;
      logprobs_kernel<T, W, decltype(tc)::value>
          <<<static_cast<unsigned>((parts + per - 1) / per), kNT, 0, s>>>(a, splits, length);
    };
    auto waves = [&](auto tc) {
      if (a.V <= 4096) with(std::integral_constant<int, 1>{}, tc);
      else with(std::integral_constant<int, 4>{}, tc);
    };
    if (a.top_k > 0) waves(std::true_type{});
    else waves(std::false_type{});
    if (splits > 1) join_kernel<T><<<static_cast<unsigned>(a.T), 64, 0, s>>>(a, splits);
  };
  if (a.dtype == BNN_I32) go(int32_t{});
  else with_real_type(a.dtype, go);
  return hipGetLastError();
}

}  // namespace bnn
