// Routing of rows to experts: scores, a balancing bias, groups, the top_k
// largest keys and their weights (bnn_route).
//
// A row's E logits lie in the registers of a wave, expert e in register e / 64
// of lane e % 64.  Keys are compared with their expert's index, so that
// equal ones go to the lowest index whatever the lanes' order.
#include <float.h>

#include "dtypes.hpp"
#include "experts.hpp"

namespace bnn {
namespace {

constexpr int kNT = 256;
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

// LP lanes per row, VPL experts per lane.
template <int LP, int VPL, bool SOFTMAX, class T>
__global__ __launch_bounds__(kNT) void route_kernel(RouteArgs a) {
  constexpr int kRows = kNT / LP;
  extern __shared__ float lds[];  // groups: [kRows][E] keys, [kRows][groups] scores
  const int ln = threadIdx.x % LP;
  const int row = threadIdx.x / LP;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kRows + row;
  const bool live = t < a.T;
  const T* src = static_cast<const T*>(a.logits) + (live ? t : a.T - 1) * a.stride;

  float p[VPL], key[VPL];
  float top = kNone;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int e = i * LP + ln;
    const float raw = e < a.E ? to_f32(src[e]) : kNone;
    // (false for NaN: such a logit is out of reach as well)
    const float z = raw > kNone ? fminf(fmaxf(raw * a.logit_scale, -FLT_MAX), FLT_MAX) : kNone;
    p[i] = z;
    top = fmaxf(top, z);
  }
  if constexpr (SOFTMAX) {
#pragma unroll
    for (int s = LP / 2; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s, LP));
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      key[i] = p[i];
      p[i] = p[i] > kNone ? expf(p[i] - top) : 0.0f;
      sum += p[i];
    }
#pragma unroll
    for (int s = LP / 2; s > 0; s >>= 1) sum += __shfl_xor(sum, s, LP);
    // (sum >= 1 where any expert is in reach)
#pragma unroll
    for (int i = 0; i < VPL; ++i) p[i] = sum > 0.0f ? p[i] / sum : 0.0f;
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      key[i] = p[i];
      p[i] = 1.0f / (1.0f + expf(-p[i]));
    }
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int e = i * LP + ln;
    const float b = a.bias && e < a.E ? a.bias[e] : 0.0f;
    const float v = p[i] + b;
    key[i] = key[i] > kNone && v > kNone ? v : kNone;
  }

  if (a.groups > 1) {
    float* keys = lds + row * a.E;
    float* scores = lds + kRows * a.E + row * a.groups;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (i * LP + ln < a.E) keys[i * LP + ln] = key[i];
    __syncthreads();
    for (int g = ln; g < a.groups; g += LP) {
      float b0 = kNone, b1 = kNone;
      for (int j = 0; j < a.per_group; ++j) {
        const float v = keys[g * a.per_group + j];
        b1 = fmaxf(b1, fminf(b0, v));
        b0 = fmaxf(b0, v);
      }
      scores[g] = a.group_top == 2 && b1 > kNone ? b0 + b1 : b0;
    }
    __syncthreads();
    // A group is kept where fewer than top_groups come before it.
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int e = i * LP + ln;
      if (e < a.E) {
        const int g = e / a.per_group;
        const float mine = scores[g];
        int before = 0;
        for (int q = 0; q < a.groups; ++q) {
          const float v = scores[q];
          before += v > mine || (v == mine && q < g) ? 1 : 0;
        }
        if (before >= a.top_groups) key[i] = kNone;
      }
    }
  }

  // k rounds: the largest key of the row, and the lowest index that has it.
  float total = 0.0f, my_w = 0.0f;
  int my_id = -1;
  for (int j = 0; j < a.k; ++j) {
    float bk = kNone, bp = 0.0f;
    int be = a.E;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (key[i] > bk) {
        bk = key[i];
        bp = p[i];
        be = i * LP + ln;
      }
#pragma unroll
    for (int s = LP / 2; s > 0; s >>= 1) {
      const float ok = __shfl_xor(bk, s, LP), op = __shfl_xor(bp, s, LP);
      const int oe = __shfl_xor(be, s, LP);
      const bool take = ok > bk || (ok == bk && oe < be);
      bk = take ? ok : bk;
      bp = take ? op : bp;
      be = take ? oe : be;
    }
    total += bp;
    if (ln == j) {
      my_id = bk > kNone ? be : -1;
      my_w = bp;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (i * LP + ln == be) key[i] = kNone;
  }
  if (live && ln < a.k) {
    if (a.renorm) my_w = total > 0.0f ? my_w / total : 0.0f;
    a.ids[t * a.k + ln] = my_id;
    a.weights[t * a.k + ln] = my_w * a.scale;
  }
}

template <int LP, int VPL, class T>
void launch_shape(const RouteArgs& a, bool softmax, hipStream_t s) {
  constexpr int kRows = kNT / LP;
  const unsigned blocks = static_cast<unsigned>((a.T + kRows - 1) / kRows);
  const size_t lds = a.groups > 1 ? size_t{kRows} * (a.E + a.groups) * sizeof(float) : 0;
  if (softmax)
    route_kernel<LP, VPL, true, T><<<blocks, kNT, lds, s>>>(a);
  else
    route_kernel<LP, VPL, false, T><<<blocks, kNT, lds, s>>>(a);
}

template <class T>
void launch_typed(const RouteArgs& a, bool softmax, hipStream_t s) {
  if (a.E <= 64)
    launch_shape<64, 1, T>(a, softmax, s);
  else if (a.E <= 256)
    launch_shape<64, 4, T>(a, softmax, s);
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
