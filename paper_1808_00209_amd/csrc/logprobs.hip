// Log probabilities of given answers, the entropy and the largest alternatives
// of a row of logits (bnn_logprobs), in one pass over them.
//
// Sums, per wave, in units of log2 with c = logit_scale * log2(e):
//   s1 = sum 2^d,  s2 = sum 2^d d,   d = c v - ref,
//   ln p_v = (c v - ref - log2 s1) ln 2,   entropy = (log2 s1 - s2 / s1) ln 2.
// ref is any number near the largest c v: it is taken from the first values and
// moved (s1 and s2 with it) only when one lies kAway above it, so that a value
// costs one fma, one exp2 and two sums, and no maximum of its own.
//
// The alternatives so far are a sorted list over the wave's lanes, one 64-bit
// key each: the value's order in the high word, the inverted index in the low
// one.  A step's 16 values per lane are looked at further only where the largest
// reaches the top_k-th key, and values are inserted one by one; where many do
// (the first step, rising rows), the bound is first raised to what top_k lanes'
// largest values reach, and what still passes is placed by counting.  Values that
// equal a full list's last key are looked at only where their index may be lower
// (4096 rows of 32768 equal fp32 values 101 us, 2990 without; random ones 101).
//
// 4096 x 131072 bf16, 8 alternatives: 193-210 us from card to card, 5.1 to 5.5
// TB/s, a large copy's rate (without alternatives 183 where it took 193): bound
// by memory, the vector ALU 91 % busy.  16384 x 1000 int32, 5 alternatives:
// 22.6-25 us, 12.7 without: a wave per row, 470 vector and 451 scalar instructions
// of which the sums are 200.  301 x 50021 fp32, 8 alternatives: 20 us, 14
// without: 1.2 rows per CU, of 16 waves that each fill a list.  One row of 65536:
// 11.6 us in two launches, chains of dependent steps.  Tried and dropped: values
// through LDS instead of 16 copies of the insertion (one row: 16.2 us against
// 14.4), the waves of a row sharing their bounds (16.1 against 13.5), the next
// step's loads ahead (no gain).
#include "dtypes.hpp"
#include "logprobs_plans.hpp"
#include "quant.hpp"
#include "wave_ops.hpp"

#include <type_traits>

namespace bnn {
namespace {

constexpr int kNT = 256;  // unless a row has more waves
constexpr int kEach = 16;          // values of a lane per step, in groups of 8
constexpr int kStep = 64 * kEach;  // of a wave
static_assert(kStep == kLogprobsStep, "the plans count in steps");
// A value this far above the reference (2^2.5 times it) moves it, so that the
// largest one's d, which log2 s1 and s2 / s1 share, has few bits before the
// point: with 16 an almost certain answer's ln p was off by up to 7e-7 and the
// entropy by 1.2e-6, now 2.3e-7.  Random rows take 0 to 2 % longer for it (4000 x
// 4096 with 8 alternatives 15.7 us : 15.4-15.7), rising ones 0.5 to 1.6 (4096 x
// 32768 210 : 207); with 1 or 2 the former is 16.1.
constexpr float kAway = 2.5f;
constexpr float kFar = 3e38f;    // the reference before there is one: minus this
constexpr float kLarge = 0x1p20f; // the quick form's references, at most
// The quick form takes integers as fp32.  Up to kExact the largest is itself, and
// a smaller one's rounding 2^-24 of its distance; beyond it c v is off by up to
// 2^-25 of itself, 2^-23 with references up to kSmall.
constexpr float kExact = 0x1p23f;
constexpr float kSmall = 4.0f;
// Integers that differ at all have no sums in common from 2^8 on: factors are cut
// to this one in them, so that no product passes fp32's range (0 * inf).
constexpr float kSharp = 0x1p90f;

struct Sums {
  double ref;
  float s1, s2;
};

// The workspace: a part's sums each, then top_k keys each.
static_assert(sizeof(Sums) == 16, "as the workspace's size counts them");
size_t part_bytes(int top_k) { return sizeof(Sums) + size_t{8} * top_k; }

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

// A wave's sorted list of keys over its lanes, the largest in lane 0 (0: none).
// bound is the key of lane top_k - 1, floor what a value's order must reach.
struct Top {
  uint32_t hi, lo;  // this lane's key
  uint32_t floor;   // uniform
  uint64_t bound;   // uniform
  uint64_t* slots;  // 64 of the wave's, in LDS

  __device__ __forceinline__ void take_bound(int top_k) {
    const uint32_t bh = __builtin_amdgcn_readlane(hi, top_k - 1);
    bound = static_cast<uint64_t>(bh) << 32 |
            static_cast<uint32_t>(__builtin_amdgcn_readlane(lo, top_k - 1));
    if (bh > floor) floor = bh;
  }

  // Whether a key (uniform) is beyond the bound, in 32-bit steps that the scalar
  // unit has.
  __device__ __forceinline__ bool beyond(uint32_t order, uint32_t low) const {
    const uint32_t bh = static_cast<uint32_t>(bound >> 32);
    return order > bh || (order == bh && low > static_cast<uint32_t>(bound));
  }

  // A key of the lanes where `is` holds, put behind the `count` ones in slots
  // (past 64: only counted).
  __device__ __forceinline__ void collect(uint64_t key, bool is, int& count) {
    const uint64_t mask = __ballot(is);
    if (!mask) return;
    const int at = count + __builtin_amdgcn_mbcnt_hi(
        static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), 0));
    if (is && at < 64) slots[at] = key;
    count += __popcll(mask);
  }

  // An empty list from the `count` <= 64 keys in slots: a key's place is the
  // number of larger ones, counted over all of them with nothing to wait for.
  __device__ __forceinline__ void fill(int count, int top_k) {
    const int lane = threadIdx.x & 63;
    const uint64_t mine = lane < count ? slots[lane] : 0;
    const uint32_t mh = static_cast<uint32_t>(mine >> 32), ml = static_cast<uint32_t>(mine);
    int place = 0;
    for (int j = 0; j < count; j += 4) {  // (keys past count are 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t other = static_cast<uint64_t>(__builtin_amdgcn_readlane(mh, j + i)) << 32 |
                               static_cast<uint32_t>(__builtin_amdgcn_readlane(ml, j + i));
        place += other > mine;
      }
    }
    if (lane < count) slots[place] = mine;
    const uint64_t key = lane < top_k && lane < count ? slots[lane] : 0;
    hi = static_cast<uint32_t>(key >> 32);
    lo = static_cast<uint32_t>(key);
    take_bound(top_k);
  }

  __device__ __forceinline__ void insert(uint64_t key, int top_k) {
    const uint64_t mine = static_cast<uint64_t>(hi) << 32 | lo;
    const int pos = __popcll(__ballot(mine > key));  // (below top_k: key > bound)
    const int lane = threadIdx.x & 63;
    const uint32_t uh = lane_before(hi), ul = lane_before(lo);
    hi = lane < pos ? hi : lane == pos ? static_cast<uint32_t>(key >> 32) : uh;
    lo = lane < pos ? lo : lane == pos ? static_cast<uint32_t>(key) : ul;
    take_bound(top_k);
  }
};

// Raises top.floor to an order that the values of at least top_k lanes reach
// (mine: a lane's largest, 0 for none): 14 bits of it below those that all lanes'
// have in common, a lower bound of the top_k-th being all that is asked (6 bits
// let too many through: 301 x 50021 34 us instead of 22).
__device__ __forceinline__ void raise_floor(Top& top, uint32_t mine, int top_k) {
  // (known as uniform: what follows is the scalar unit's)
  const uint32_t most = __builtin_amdgcn_readfirstlane(wave_max(mine));
  const uint32_t least = __builtin_amdgcn_readfirstlane(wave_min(mine ? mine : ~0u));
  const int own = most == least ? 0 : 32 - __builtin_clz(most ^ least);  // bits
  uint32_t at = own < 32 ? most >> own << own : 0;
  if (__popcll(__ballot(mine >= at && mine != 0)) < top_k) return;
  for (int b = own - 1; b >= 0 && b >= own - 14; --b) {
    const uint32_t next = at | 1u << b;
    if (__popcll(__ballot(mine >= next)) >= top_k) at = next;
  }
  if (at > top.floor) top.floor = at;
}

// SAFE: the reference is the largest value itself and differences are taken
// before the factor, of integers as integers, for rows whose c v pass 2^20 (or
// pass kSmall with integers beyond kExact), rows without a value in reach and
// rows with NaN or infinity (whose quick sums end as 0, NaN or infinity).
template <bool SAFE, class R>
struct Scan {
  static constexpr bool kInts = std::is_same<R, int32_t>::value;
  using Ref = std::conditional_t<SAFE, R, float>;
  float c;  // (of integers at most kSharp)
  Ref ref;
  float s1, s2;

  __device__ __forceinline__ void start(float factor) {
    c = kInts ? __builtin_fminf(factor, kSharp) : factor;
    if constexpr (!SAFE) ref = -kFar;
    else if constexpr (kInts) ref = INT32_MIN;
    else ref = -__builtin_inff();
    s1 = s2 = 0.0f;
  }
  // c (from - to) of integers, from <= to.
  __device__ __forceinline__ float fall(int32_t from, int32_t to) const {
    return -static_cast<float>(static_cast<uint32_t>(to) - static_cast<uint32_t>(from)) * c;
  }
  // (SAFE: of a value that is not above the reference)
  __device__ __forceinline__ float delta(R v) const {
    if constexpr (!SAFE) return __builtin_fmaf(static_cast<float>(v), c, -ref);
    else if constexpr (kInts) return fall(v, ref);
    else return v == -__builtin_inff() ? v : (v - ref) * c;
  }
  // The reference for values up to m (of each lane that has some).
  __device__ __forceinline__ void refer(R m, bool some) {
    if constexpr (SAFE) {
      if (__any(some && m > ref)) {
        const R next = wave_max(some ? m : ref);
        if constexpr (kInts) move_to(next, fall(ref, next));
        else move_to(next, (ref - next) * c);
      }
    } else {
      const float fm = some ? static_cast<float>(m) : -__builtin_inff();
      if (__any(__builtin_fmaf(fm, c, -ref) > kAway)) {
        const float top = wave_max(fm), next = top * c;
        // (a quick reference's own rounding must not count: 2^-5 at most; nor an
        // integer's: of 2^-24 c v, where one beyond kExact is asked for)
        const float most = kInts && __builtin_fabsf(top) > kExact ? kSmall : kLarge;
        if (!(__builtin_fabsf(next) <= most)) s1 = __builtin_nanf("");
        move_to(next, ref - next);
      }
    }
  }
  __device__ __forceinline__ void move_to(Ref next, float move) {
    move = s1 == 0.0f ? -1e4f : __builtin_fmaxf(move, -1e4f);
    const float f = exp2_of(move);
    s2 = f * __builtin_fmaf(move, s1, s2);
    s1 *= f;
    ref = next;
  }
  // The first n of v (8 and more: all).  FINITE: no value is -inf.
  template <bool FINITE>
  __device__ __forceinline__ void add(const R (&v)[8], int n) {
    float e[8], d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      d[i] = i < n ? delta(v[i]) : -__builtin_inff();
      e[i] = exp2_of(d[i]);
      if (!FINITE) d[i] = __builtin_fmaxf(d[i], -200.0f);  // (0 * -inf)
    }
    s1 += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    float t = e[0] * d[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) t = __builtin_fmaf(e[i], d[i], t);
    s2 += t;
  }
  // (a quick reference with a factor beyond kSharp is 0)
  __device__ __forceinline__ Sums total(float factor) const {
    return {SAFE ? static_cast<double>(ref) * factor : static_cast<double>(ref), wave_sum(s1),
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

// Values [begin, end) of a row, by wave `wave` of W.
template <class T, bool SAFE, bool TOP, int W>
__device__ __forceinline__ Sums scan(const T* row, int begin, int end, int wave, float c, int top_k,
                                     Top& top) {
  using R = typename RawOf<T>::type;
  constexpr bool kInts = std::is_same<R, int32_t>::value;
  constexpr int kGroups = kEach / 8;
  const int lane = threadIdx.x & 63;
  Scan<SAFE, R> sc;
  sc.start(c);
  // A step: group g of a lane's 8 values starts at index at + 512 g + 8 lane.
  // What lies past the row's end is -inf; integers have no such value, so there
  // `n` says how many of each group are in the row: all (kAll), all or none
  // (kWhole), or some (kSome).
  constexpr int kAll = 0, kWhole = 1, kSome = 2;
  auto step = [&](const R (&v)[kEach], int at, const int (&n)[kGroups], auto part) {
    constexpr int kPart = kInts ? decltype(part)::value : kAll;
    auto in = [&](int i) { return kPart == kAll || (kPart == kWhole ? n[i / 8] > 0 : i % 8 < n[i / 8]); };
    R m = v[0];
    if constexpr (kInts) {  // (beyond 2^24 their order is not that of fp32)
#pragma unroll
      for (int i = 1; i < kEach; ++i) m = m > v[i] ? m : v[i];
    } else {
#pragma unroll
      for (int i = 1; i < kEach; ++i) m = __builtin_fmaxf(m, v[i]);
    }
    const bool some = kPart == kAll || n[0] > 0;  // (past the end: the least integer)
    sc.refer(m, some);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      if (kPart == kWhole && n[g] <= 0) continue;
      R f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = v[8 * g + i];
      sc.template add<kInts && kPart != kSome>(f, kPart == kSome ? n[g] : 8);
    }
    if constexpr (TOP) {
      // (a full list of earlier values: one that is equal to its last is behind)
      const uint32_t last = static_cast<uint32_t>(top.bound >> 32);
      if (top.bound != 0 && top.floor == last && last != ~0u && ~static_cast<uint32_t>(top.bound) < static_cast<uint32_t>(at))
        top.floor = last + 1;
      const uint32_t mo = some ? order_of(m) : 0u;
      const uint64_t reach = __ballot(some && mo >= top.floor);
      if (reach) {
        if (__popcll(reach) > 12) raise_floor(top, mo, top_k);
        R floor;
        value_of(top.floor, floor);
        auto passes = [&](int i) { return v[i] >= floor && in(i); };
        auto index_of = [&](int i, int l) { return static_cast<uint32_t>(at + i / 8 * 512 + 8 * l + i % 8); };
        // (an empty list of few is filled sooner by inserting: 16384 x 1000, 5
        // alternatives 23.4 us : 25.6; 301 x 50021, 8 alternatives 27 : 22)
        if (top_k > 6 && top.bound == 0) {  // (not full: most often, empty)
          const bool empty = __builtin_amdgcn_readlane(top.hi | top.lo, 0) == 0;
          int count = 0;
          if (empty) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
              top.collect(static_cast<uint64_t>(order_of(v[i])) << 32 | static_cast<uint32_t>(~index_of(i, lane)),
                          passes(i), count);
          }
          if (empty && count <= 64) {
            top.fill(count, top_k);
            return;
          }
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          uint64_t mask = __ballot(passes(i));
          if (!mask) continue;
          if (__popcll(mask) > 8) {  // (equal values: only those of lower index)
            const uint64_t mine = static_cast<uint64_t>(order_of(v[i])) << 32 |
                                  static_cast<uint32_t>(~index_of(i, lane));
            mask &= __ballot(mine > top.bound);
          }
          while (mask) {
            const int l = __builtin_ctzll(mask);
            mask &= mask - 1;
            const uint32_t o = order_of(__builtin_bit_cast(
                R, __builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, v[i]), l)));
            const uint32_t low = ~index_of(i, l);
            if (top.beyond(o, low)) {
              top.insert(static_cast<uint64_t>(o) << 32 | low, top_k);
              value_of(top.floor, floor);
            }
          }
        }
      }
    }
  };
  T past;
  if constexpr (kInts) past = INT32_MIN;
  else past = static_cast<T>(-__builtin_inff());
  R v[kEach];
  int n[kGroups] = {};
  auto take = [&](const Eight<T> (&e)[kGroups]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = static_cast<R>(e[i / 8].v[i % 8]);
  };
  int at = begin + wave * kStep;
  for (; at + kStep <= end; at += W * kStep) {
    Eight<T> e[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) e[g] = load8(row + at + 512 * g + 8 * lane);
    take(e);
    step(v, at, n, std::integral_constant<int, kAll>{});
  }
  if (at < end) {
    Eight<T> e[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int first = at + 512 * g + 8 * lane;
      n[g] = end - first;
#pragma unroll
      for (int i = 0; i < 8; ++i) e[g].v[i] = past;
      if (n[g] >= 8) {
        e[g] = load8(row + first);
      } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
          if (i < n[g]) e[g].v[i] = row[first + i];
      }
    }
    take(e);
    if (kInts && (end - at) % 8 == 0) step(v, at, n, std::integral_constant<int, kWhole>{});
    else step(v, at, n, std::integral_constant<int, kSome>{});
  }
  return sc.total(c);
}

// A wave's sums: in fp32's range by the quick form, or else by the safe one.
template <class T, bool TOP, int W>
__device__ __forceinline__ Sums wave_part(const T* row, int begin, int end, int wave, float c, int top_k,
                                          Top& top) {
  Sums s = scan<T, false, TOP, W>(row, begin, end, wave, c, top_k, top);
  if (!(s.s1 > 0.0f && s.s1 < __builtin_inff()))
    s = scan<T, true, false, W>(row, begin, end, wave, c, top_k, top);
  return s;
}

// A lane's keys out of `count` (0: none): these in registers, others are read
// again.
constexpr int kHeld = 4;
struct Held {
  uint64_t key[kHeld];
};
__device__ __forceinline__ Held hold_keys(const uint64_t* keys, int count) {
  Held h;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = 64 * j + static_cast<int>(threadIdx.x & 63);
    h.key[j] = i < count ? keys[i] : 0;
  }
  return h;
}

// The top_k largest of `count` keys, by one wave.
__device__ __forceinline__ Top select_keys(const Held& h, const uint64_t* keys, int count, int top_k,
                                           uint64_t* slots) {
  const int lane = threadIdx.x & 63;
  uint32_t most = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const uint32_t o = static_cast<uint32_t>(h.key[j] >> 32);
    most = most > o ? most : o;
  }
  for (int i = 64 * kHeld + lane; i < count; i += 64) {
    const uint32_t o = static_cast<uint32_t>(keys[i] >> 32);
    most = most > o ? most : o;
  }
  Top top = {0, 0, 0, 0, slots};
  raise_floor(top, most, top_k);
  int collected = 0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    top.collect(h.key[j], h.key[j] != 0 && static_cast<uint32_t>(h.key[j] >> 32) >= top.floor, collected);
  for (int i0 = 64 * kHeld; i0 < count; i0 += 64) {
    const uint64_t key = i0 + lane < count ? keys[i0 + lane] : 0;
    top.collect(key, key != 0 && static_cast<uint32_t>(key >> 32) >= top.floor, collected);
  }
  if (collected <= 64) {
    top.fill(collected, top_k);
    return top;
  }
  for (int i0 = 0; i0 < count; i0 += 64) {  // (many equal ones)
    const uint64_t key = i0 + lane < count ? keys[i0 + lane] : 0;
    const uint32_t hi = static_cast<uint32_t>(key >> 32), lo = static_cast<uint32_t>(key);
    uint64_t mask = __ballot(hi >= top.floor && key > top.bound);
    while (mask) {
      const int l = __builtin_ctzll(mask);
      mask &= mask - 1;
      const uint32_t o = __builtin_amdgcn_readlane(hi, l), low = __builtin_amdgcn_readlane(lo, l);
      if (top.beyond(o, low)) top.insert(static_cast<uint64_t>(o) << 32 | low, top_k);
    }
  }
  return top;
}

// Sums over the wave's lanes.
__device__ __forceinline__ Sums lanes_joined(Sums s) {
  const double ref = wave_max(s.s1 == 0.0f ? -__builtin_inf() : s.ref);
  if (s.s1 == 0.0f) s.ref = ref;
  // (a part with NaN for sums: NaN, whatever its reference)
  const float move = ref > -__builtin_inf() ? fmaxf(static_cast<float>(s.ref - ref), -1e4f) : 0.0f;
  const float f = exp2_of(move);
  return {ref > -__builtin_inf() ? ref : 0.0, wave_sum(f * s.s1),
          wave_sum(f * __builtin_fmaf(move, s.s1, s.s2))};
}

// The first 64 of a row's given answers, a lane's: asked for early, since the
// logit waits for the id (ids first, then `gather`).
template <class T>
struct Given {
  using R = typename RawOf<T>::type;
  int id = -1;
  R v = 0;
  __device__ __forceinline__ void ask(const LogprobsArgs& a, int64_t t) {
    const int lane = threadIdx.x & 63;
    if (lane < a.n) id = a.ids[t * a.n + lane];
  }
  __device__ __forceinline__ void gather(const LogprobsArgs& a, int64_t t) {
    if (id >= 0 && id < a.V) v = static_cast<R>(static_cast<const T*>(a.logits)[t * a.stride + id]);
  }
};

// A row's outputs from its sums and (lane j: the j-th) keys, by one wave.
template <class T>
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int64_t t, const Sums& s,
                                          uint64_t key, float c, Given<T> given) {
  using R = typename RawOf<T>::type;
  constexpr double kLn2 = 0.693147180559945309417;
  const int lane = threadIdx.x & 63;
  const bool none = s.s1 == 0.0f, bad = !(s.s1 < __builtin_inff());
  // (the largest value's part is 1 or more, but for the reference's rounding)
  const float ls = __builtin_amdgcn_logf(s.s1);
  const float ref = static_cast<float>(s.ref);
  const bool quick = static_cast<double>(ref) == s.ref && __builtin_fabsf(ref) <= kLarge;
  const float nan = __builtin_nanf("");
  auto ln_p = [&](R v) {
    if (std::is_same<R, float>::value && static_cast<float>(v) == -__builtin_inff())
      return -__builtin_inff();
    const float f = static_cast<float>(v), d = __builtin_fmaf(f, c, -ref);
    const bool as_is = std::is_same<R, float>::value || __builtin_fabsf(f) < 0x1p24f;
    const float lp = quick && as_is && __builtin_fabsf(d) < 1e30f
        ? (d - ls) * static_cast<float>(kLn2)
        : static_cast<float>((static_cast<double>(v) * c - s.ref - static_cast<double>(ls)) * kLn2);
    return lp > 0.0f ? 0.0f : lp;  // (roundings may pass 0)
  };
  auto not_below_0 = [](float h) { return h < 0.0f ? 0.0f : h; };
  if (a.entropy && lane == 0)
    a.entropy[t] = bad ? nan : none ? 0.0f
        : not_below_0((ls - s.s2 / s.s1) * static_cast<float>(kLn2));
  for (int j = lane; j < a.n; j += 64) {
    if (j >= 64) {
      given.id = a.ids[t * a.n + j];
      given.gather(a, t);
    }
    const bool there = given.id >= 0 && given.id < a.V;
    a.logp[t * a.n + j] = !there || (none && !bad) ? -__builtin_inff() : bad ? nan : ln_p(given.v);
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
__global__ __launch_bounds__(W > 4 ? W * 64 : kNT) void logprobs_kernel(LogprobsArgs a, int splits,
                                                                        int length) {
  using R = typename RawOf<T>::type;
  __shared__ Sums sums[W];
  __shared__ uint64_t keys[W * BNN_MAX_ALTERNATIVES];
  __shared__ uint64_t slots[W > 4 ? W : 4][64];
  constexpr int kParts = W > 4 ? 1 : 4 / W;  // of a workgroup
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = W == 1 ? 0 : id;
  const int64_t part = static_cast<int64_t>(blockIdx.x) * kParts + (W == 1 ? id : 0);
  // (split rows: T < kFull, so that parts fit 32 bits)
  const int64_t t = splits == 1 ? part : static_cast<uint32_t>(part) / static_cast<uint32_t>(splits);
  if (t >= a.T) return;
  const int begin = static_cast<int>(part - t * splits) * length;
  const int end = min(begin + length, a.V);
  const T* row = static_cast<const T*>(a.logits) + t * a.stride;
  const float c = factor_of(a.scale);
  Top top = {0, 0, kFloor<R>, 0, slots[id]};
  Given<T> given;
  if (splits == 1 && wave == 0) given.ask(a, t);
  Sums s = wave_part<T, TOP, W>(row, begin, end, wave, c, a.top_k, top);
  if (splits == 1 && wave == 0) given.gather(a, t);
  if constexpr (W > 1) {
    if (lane == 0) sums[wave] = s;
    if (TOP && lane < a.top_k) keys[wave * a.top_k + lane] = static_cast<uint64_t>(top.hi) << 32 | top.lo;
    __syncthreads();
    if (wave != 0) return;
    s = lane < W ? sums[lane < W ? lane : 0] : Sums{0.0, 0.0f, 0.0f};
    s = lanes_joined(s);
    if constexpr (TOP) top = select_keys(hold_keys(keys, W * a.top_k), keys, W * a.top_k, a.top_k, slots[0]);
  }
  const uint64_t key = static_cast<uint64_t>(top.hi) << 32 | top.lo;
  if (splits == 1) {
    write_row<T>(a, t, s, key, c, given);
  } else {
    Sums* all = static_cast<Sums*>(a.workspace);
    if (lane == 0) all[part] = s;
    if (TOP && lane < a.top_k)
      reinterpret_cast<uint64_t*>(all + a.T * splits)[part * a.top_k + lane] = key;
  }
}

// A row's parts put together, by one wave.
template <class T>
__global__ __launch_bounds__(64) void join_kernel(LogprobsArgs a, int splits) {
  __shared__ uint64_t slots[64];
  const int64_t t = blockIdx.x;
  const Sums* all = static_cast<const Sums*>(a.workspace);
  const uint64_t* keys = reinterpret_cast<const uint64_t*>(all + a.T * splits) + t * splits * a.top_k;
  const int lane = threadIdx.x;
  // everything is asked for before anything is waited for
  Given<T> given;
  given.ask(a, t);
  Sums s = lane < splits ? all[t * splits + lane] : Sums{0.0, 0.0f, 0.0f};
  const Held held = hold_keys(keys, splits * a.top_k);
  __builtin_amdgcn_sched_barrier(0);
  given.gather(a, t);
  s = lanes_joined(s);
  for (int p0 = 64; p0 < splits; p0 += 64) {
    Sums more = {0.0, 0.0f, 0.0f};
    if (p0 + lane < splits) more = all[t * splits + p0 + lane];
    s = joined(s, lanes_joined(more));
  }
  Top top = {};
  if (a.top_k > 0) top = select_keys(held, keys, splits * a.top_k, a.top_k, slots);
  write_row<T>(a, t, s, static_cast<uint64_t>(top.hi) << 32 | top.lo, factor_of(a.scale), given);
}

}  // namespace

size_t logprobs_workspace(int64_t T, int32_t V, int32_t top_k) {
  return static_cast<size_t>(logprobs_parts(T, V)) * part_bytes(top_k);
}

hipError_t launch_logprobs(const LogprobsArgs& a, hipStream_t s) {
  const LogprobsPlan plan = logprobs_plan(a.T, a.V);
  const int splits = plan.splits;
  auto go = [&](auto t) {
    using T = decltype(t);
    auto with = [&](auto wc, auto tc) {
      constexpr int W = decltype(wc)::value;
      constexpr int per = W > 4 ? 1 : 4 / W;
      const int64_t parts = a.T * splits;
      logprobs_kernel<T, W, decltype(tc)::value>
          <<<static_cast<unsigned>((parts + per - 1) / per), W > 4 ? W * 64 : kNT, 0, s>>>(a, splits, plan.length);
    };
    auto waves = [&](auto tc) {
      if (plan.waves == 1) with(std::integral_constant<int, 1>{}, tc);
      else if (plan.waves == 16) with(std::integral_constant<int, 16>{}, tc);
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
