// Routing of rows to experts: scores, a balancing bias, groups, the top_k
// largest keys and their weights (bnn_route).
//
// A row's E logits lie in the registers of LP lanes, VPL consecutive experts
// in each.  Every lane keeps its four largest keys, in order (v_med3_f32 puts a
// key in its place, an instruction for each of the four).  A round takes the
// largest of the row's heads, as whole numbers of the keys' order (DPP steps
// within 16 lanes; of equal ones the lowest lane's, whose experts come first),
// and its lane moves up, noting the key and how many equal ones it gave before.
// A lane that gave four looks through its keys again.  Which expert of the lane
// a key belongs to is found at the end, once for each of the top_k, from the
// keys in LDS.  The weights are computed again for the chosen experts alone.
//
// 65521 rows of 256 experts in 8 groups, sigmoid scores and a bias: 67 MB of
// logits, 14 us at 5.1 TB/s; 24.9 us, the vector ALU busy in three quarters of
// them (854 instructions for four rows; with the experts' indices carried along
// in the low bits of doubles 1030 and 27.7 us).  A wave per row with shuffles
// took 139 us.
#include <float.h>

#include <type_traits>

#include "dtypes.hpp"
#include "experts.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;
constexpr int kKeep = 4;             // experts that a lane holds ready
constexpr float kNone = -INFINITY;  // the key of an expert out of reach

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* ids;
  float* weights;
  int64_t stride;
  int32_t T, E, k, groups, per_group, top_groups, group_top, renorm;
  float scale, logit_scale;
};

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  const int v = __float_as_int(x);
  return __int_as_float(__builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  const int v = static_cast<int>(x);
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false));
}

// f over the LP lanes of a row; every lane gets the result.  f commutes, so
// all lanes get the same bits.
template <int LP, class V, class F>
__device__ __forceinline__ V row_reduce(V x, F f) {
  x = f(x, dpp<0xB1>(x));   // quad_perm [1,0,3,2]
  x = f(x, dpp<0x4E>(x));   // quad_perm [2,3,0,1]
  x = f(x, dpp<0x141>(x));  // row_half_mirror: the other quad of 8 lanes
  x = f(x, dpp<0x140>(x));  // row_mirror: the other 8 of 16
#pragma unroll
  for (int s = 16; s < LP; s *= 2) x = f(x, __shfl_xor(x, s));
  return x;
}

// exp(z) within a few units of the last place for z in [-1000, 1000]: exp2 of
// the rounded z log2(e) times 1 + the rest; 0 and infinity outside the normal
// range.
__device__ __forceinline__ float exp_of(float z) {
  constexpr float kL = 1.44269502162933349609375f;      // log2(e) rounded
  constexpr float kLlo = 1.925963033500011079e-8f;      // log2(e) - kL
  constexpr float kLn2 = 0.693147180559945309417f;
  const float t = z * kL;
  const float rest = fmaf(z, kLlo, fmaf(z, kL, -t));
  return __builtin_amdgcn_exp2f(t) * fmaf(rest, kLn2, 1.0f);
}

// z within [-limit, limit].
__device__ __forceinline__ float clamped(float z, float limit) {
  return __builtin_amdgcn_fmed3f(z, -limit, limit);
}

// The larger of two numbers that are not NaN (fmaxf quiets signalling ones
// first, an instruction for each operand).
__device__ __forceinline__ float larger(float x, float y) {
  return __builtin_amdgcn_fmed3f(x, y, INFINITY);
}

// A logit in reach (not -inf or NaN) as its score; top and 1 / sum of the
// row's softmax.  (A sigmoid's argument beyond +-1000 gives 0 or 1 as it is.)
template <bool SOFTMAX>
__device__ __forceinline__ float score(float raw, float scale, float top, float inv_sum) {
  if constexpr (SOFTMAX)
    return exp_of(clamped(clamped(raw * scale, FLT_MAX) - top, 1000.0f)) * inv_sum;
  return __builtin_amdgcn_rcpf(1.0f + exp_of(clamped(-(raw * scale), 1000.0f)));
}

// A key as a whole number of the same order, and back.
__device__ __forceinline__ uint32_t ordered(float key) {
  const uint32_t b = __float_as_uint(key);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u ^ (static_cast<uint32_t>(~static_cast<int32_t>(u) >> 31) | 0x80000000u));
}
constexpr uint32_t kNoneBits = 0x007FFFFFu;  // ordered(kNone)

// LP lanes per row, VPL experts per lane.
template <int LP, int VPL, bool SOFTMAX, class T>
__global__ __launch_bounds__(kNT) void route_kernel(RouteArgs a) {
  constexpr int kRows = kNT / LP;
  extern __shared__ __attribute__((aligned(8))) float lds[];  // groups only
  const int ln = threadIdx.x % LP;
  const int row = threadIdx.x / LP;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + row;
  const bool live = t < a.T;
  const T* src = static_cast<const T*>(a.logits) + (live ? t : a.T - 1) * a.stride;
  const int e0 = ln * VPL;

  T raw[VPL];
  float key[VPL];  // first the logits
  if (e0 + VPL <= a.E) {
    __builtin_memcpy(raw, src + e0, sizeof(raw));
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = to_f32(raw[i]);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = e0 + i < a.E ? to_f32(src[e0 + i]) : kNone;
  }
  float top = 0.0f, inv_sum = 1.0f;
  if constexpr (SOFTMAX) {
    top = kNone;
    float ex[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {  // (false for NaN: out of reach as well)
      ex[i] = key[i] > kNone ? clamped(key[i] * a.logit_scale, FLT_MAX) : kNone;
      top = fmaxf(top, ex[i]);
    }
    top = row_reduce<LP>(top, [](float x, float y) { return fmaxf(x, y); });
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {  // (0 where out of reach)
      ex[i] = exp_of(clamped(ex[i] - top, 1000.0f));
      sum += ex[i];
    }
    sum = row_reduce<LP>(sum, [](float x, float y) { return x + y; });
    // (sum >= 1 where any expert is in reach)
    inv_sum = sum > 0.0f ? __builtin_amdgcn_rcpf(sum) : 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = key[i] > kNone ? ex[i] * inv_sum : kNone;
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const float v = score<false>(key[i], a.logit_scale, 0.0f, 0.0f);
      key[i] = key[i] > kNone ? v : kNone;
    }
  }
  if (a.bias) {
    float b[VPL];
    if (e0 + VPL <= a.E) {
      __builtin_memcpy(b, a.bias + e0, sizeof(b));
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) b[i] = e0 + i < a.E ? a.bias[e0 + i] : 0.0f;
    }
    // (the larger of NaN and kNone is kNone)
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = fmaxf(key[i] + b[i], kNone);
  }

  if (a.groups > 1) {
    // Groups of whole lanes: the two largest keys of every lane meet in LDS;
    // other groups: all keys.
    const bool whole = a.per_group % VPL == 0;
    float2* pairs = reinterpret_cast<float2*>(lds) + row * (LP + 1);
    float* keys = lds + row * a.E;
    float* scores = lds + kRows * (whole ? 2 * (LP + 1) : a.E) + row * 2 * a.groups;
    float* kept = scores + a.groups;
    if (whole) {
      float2 b = {kNone, kNone};
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        b.y = __builtin_amdgcn_fmed3f(key[i], b.x, b.y);
        b.x = larger(b.x, key[i]);
      }
      pairs[ln] = b;
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (e0 + i < a.E) keys[e0 + i] = key[i];
    }
    __syncthreads();
    for (int g = ln; g < a.groups; g += LP) {
      float b0 = kNone, b1 = kNone;
      if (whole) {
        const int n = a.per_group / VPL;
        for (int j = 0; j < n; ++j) {
          const float2 v = pairs[g * n + j];
          b1 = larger(__builtin_amdgcn_fmed3f(b0, b1, v.x), v.y);
          b0 = larger(b0, v.x);
        }
      } else {
        for (int j = 0; j < a.per_group; ++j) {
          const float v = keys[g * a.per_group + j];
          b1 = __builtin_amdgcn_fmed3f(b0, b1, v);
          b0 = larger(b0, v);
        }
      }
      // (-inf is the score of a group without any key in reach)
      scores[g] = a.group_top == 2 && b1 > kNone ? fmaxf(b0 + b1, -FLT_MAX) : b0;
    }
    __syncthreads();
    // A group is kept where fewer than top_groups come before it.
    for (int g = ln; g < a.groups; g += LP) {
      const float mine = scores[g];
      int before = 0;
      for (int q = 0; q < a.groups; ++q) {
        const float v = scores[q];
        before += v > mine || (v == mine && q < g) ? 1 : 0;
      }
      kept[g] = before < a.top_groups ? 1.0f : 0.0f;
    }
    __syncthreads();
    int g = e0 / a.per_group, at = e0 - g * a.per_group;
    float on = g < a.groups ? kept[g] : 0.0f;
    if (whole) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) key[i] = on != 0.0f ? key[i] : kNone;
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        key[i] = on != 0.0f ? key[i] : kNone;
        if (++at == a.per_group) {
          at = 0;
          ++g;
          on = g < a.groups ? kept[g] : 0.0f;
        }
      }
    }
  }

  // The lane's largest keys; where it looks again, without those above `last`
  // and the first `skip` of those equal to it.
  uint32_t u[kKeep];
  auto largest = [&](auto again, float last, int skip) {
    float best[kKeep];
#pragma unroll
    for (int q = 0; q < kKeep; ++q) best[q] = kNone;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      float v = key[i];
      if constexpr (decltype(again)::value) {
        const bool same = v == last;
        v = v < last || (same && skip <= 0) ? v : kNone;
        skip -= same ? 1 : 0;
      }
#pragma unroll
      for (int q = kKeep - 1; q > 0; --q)
        best[q] = __builtin_amdgcn_fmed3f(v, best[q - 1], best[q]);
      best[0] = larger(v, best[0]);
    }
#pragma unroll
    for (int q = 0; q < kKeep; ++q) u[q] = ordered(best[q]);
  };
  largest(std::false_type{}, 0.0f, 0);
  constexpr int kStride = VPL + 4;  // LDS floats per lane: 16-byte rows, spread over the banks
  __shared__ __attribute__((aligned(16))) float all[kRows][LP * kStride];
#pragma unroll
  for (int i = 0; i < VPL; i += 4)
    *reinterpret_cast<float4*>(&all[row][ln * kStride + i]) =
        float4{key[i], key[i + 1], key[i + 2], key[i + 3]};
  // A round takes the largest head of the row; of equal ones the lowest lane's,
  // whose experts come first.  Its lane notes itself, the key, and how many
  // equal ones it gave before, and moves up.
  __shared__ uint2 chosen[kRows][BNN_MAX_TOP_K];
  const uint64_t my_row =
      LP == 64 ? ~uint64_t{0}
               : ((uint64_t{1} << (LP & 63)) - 1) << ((threadIdx.x & 63) / LP * LP);
  int given = 0, same = 0;
  uint32_t last = 0;
  for (int j = 0; j < a.k; ++j) {
    if (VPL > kKeep && __ballot(given == kKeep)) {
      uint32_t held[kKeep];
#pragma unroll
      for (int q = 0; q < kKeep; ++q) held[q] = u[q];
      largest(std::true_type{}, unordered(last), same + 1);
#pragma unroll
      for (int q = 0; q < kKeep; ++q) u[q] = given == kKeep ? u[q] : held[q];
      given = given == kKeep ? 0 : given;
    }
    const uint32_t best =
        row_reduce<LP>(u[0], [](uint32_t x, uint32_t y) { return x > y ? x : y; });
    bool mine = u[0] == best;
    uint64_t heads = __ballot(mine);
    if (__popcll(heads) != 64 / LP) {  // (else one in every row)
      heads &= my_row;
      mine = mine && __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(heads >> 32),
                                               __builtin_amdgcn_mbcnt_lo(
                                                   static_cast<uint32_t>(heads), 0)) == 0;
    }
    if (mine) {
      same = best == last ? same + 1 : 0;
      last = best;
      chosen[row][j] = uint2{best, static_cast<uint32_t>(ln | same << 8)};
#pragma unroll
      for (int q = 0; q + 1 < kKeep; ++q) u[q] = u[q + 1];
      u[kKeep - 1] = 0;
      ++given;
    }
  }
  // (a row's lanes are of one wave, whose LDS operations keep their order)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // Lane j finds the j-th expert among those of the lane that gave it.
  int my_id = -1;
  if (ln < a.k) {
    const uint2 note = chosen[row][ln];
    const float mine = unordered(note.x);
    const int from = static_cast<int>(note.y & 255u);
    int before = static_cast<int>(note.y >> 8), at = 0;
    float v[VPL];
#pragma unroll
    for (int i = 0; i < VPL; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(&all[row][from * kStride + i]);
      v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
    }
    if (__ballot(before > 0)) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        at = v[i] == mine && before == 0 ? i : at;
        before -= v[i] == mine ? 1 : 0;
      }
    } else {
#pragma unroll
      for (int i = VPL - 1; i >= 0; --i) at = v[i] == mine ? i : at;
    }
    if (note.x > kNoneBits) my_id = from * VPL + at;
  }
  float w = my_id >= 0 ? score<SOFTMAX>(to_f32(src[my_id]), a.logit_scale, top, inv_sum) : 0.0f;
  if (a.renorm) {
    const float total = row_reduce<LP>(w, [](float x, float y) { return x + y; });
    w = total > 0.0f ? w / total : 0.0f;
  }
  if (live && ln < a.k) {
    a.ids[t * a.k + ln] = my_id;
    a.weights[t * a.k + ln] = w * a.scale;
  }
}

template <int LP, int VPL, class T>
void launch_shape(const RouteArgs& a, bool softmax, hipStream_t s) {
  constexpr int kRows = kNT / LP;
  const unsigned blocks = static_cast<unsigned>((a.T + kRows - 1) / kRows);
  const int keys = a.per_group % VPL == 0 ? 2 * (LP + 1) : a.E;
  const size_t lds = a.groups > 1 ? size_t{kRows} * (keys + 2 * a.groups) * sizeof(float) : 0;
  if (softmax)
    route_kernel<LP, VPL, true, T><<<blocks, kNT, lds, s>>>(a);
  else
    route_kernel<LP, VPL, false, T><<<blocks, kNT, lds, s>>>(a);
}

template <class T>
void launch_typed(const RouteArgs& a, bool softmax, hipStream_t s) {
  if (a.E <= 64)
    launch_shape<16, 4, T>(a, softmax, s);
  else if (a.E <= 128)
    launch_shape<16, 8, T>(a, softmax, s);
  else if (a.E <= 256)
    launch_shape<16, 16, T>(a, softmax, s);
  else
    launch_shape<64, 16, T>(a, softmax, s);
}

}  // namespace

hipError_t launch_route(const bnn_route_desc& d, int64_t T, const void* logits, int64_t stride,
                        const float* bias, int32_t* ids, float* weights, hipStream_t s) {
  RouteArgs a;
  a.logits = logits;
  a.bias = bias;
  a.ids = ids;
  a.weights = weights;
  a.stride = stride;
  a.T = static_cast<int32_t>(T);
  a.E = d.E;
  a.k = d.top_k;
  a.groups = d.groups;
  a.per_group = d.E / d.groups;
  a.top_groups = d.top_groups;
  a.group_top = d.group_top;
  a.renorm = d.renorm;
  a.scale = d.scale;
  a.logit_scale = d.logit_scale;
  const bool softmax = d.score == BNN_SCORE_SOFTMAX;
  if (d.dtype == BNN_I32)
    launch_typed<int32_t>(a, softmax, s);
  else
    with_real_type(d.dtype, [&](auto v) { launch_typed<decltype(v)>(a, softmax, s); });
  return hipGetLastError();
}

}  // namespace bnn
