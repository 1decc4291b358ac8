// How the log probabilities' kernel (logprobs.hip) spreads rows over waves and
// workgroups: rules on their number and length, as host functions.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace bnn {

constexpr int kLogprobsStep = 1024;  // values of a wave's step

// From kFull rows on, each is one workgroup's (or wave's): 200 x 50021 fp32 15.4
// us, in parts and joined 19.3; 255 x 65536 bf16 17.3 : 21.3, but 128 x 131072
// 23.8 : 20.9.  Fewer are split, if there are 4096 values for each of three parts
// (rounded up: a row of 8193 goes in three of 3072), so that a part's four waves
// have a step each (one row of 65536: 12 us; as one workgroup of 16 waves 22; 64 x
// 8000 in two parts 10.3, whole 9.0).  Long rows that leave CUs with one or two
// workgroups go to 16 waves (301 x 50021: 20 us, 4 waves 24).  A row is one wave's
// if it has one step, or up to four with rows for all waves (4000 x 4096 bf16 16.2
// us, four waves 18.9; 1000 x 4096 11.1 : 8.6).
constexpr int kFull = 160;
constexpr int kLongFew = 512;    // rows, below which long ones have 16 waves
constexpr int kParts = 1024;     // parts that fill the card
constexpr int kSplitBy = 4 * kLogprobsStep;

inline int64_t logprobs_most_splits(int32_t V) {
  const int64_t n = (V + kSplitBy - 1) / kSplitBy;
  return n < 3 ? 1 : n;
}

struct LogprobsPlan {
  int waves;   // 1, 4 or 16, of a row or of each of its parts
  int splits;  // parts of a row
  int length;  // values of a part, a whole number of steps
};

// T >= 1 rows of V values.
inline LogprobsPlan logprobs_plan(int64_t T, int32_t V) {
  LogprobsPlan p = {4, 1, 0};
  if (T < kFull) {
    const int64_t want = (kParts + T - 1) / T, most = logprobs_most_splits(V);
    p.splits = static_cast<int>(want < most ? want : most);
  }
  p.length = ((V + p.splits - 1) / p.splits + kLogprobsStep - 1) / kLogprobsStep * kLogprobsStep;
  if (V <= kLogprobsStep || (V <= 4 * kLogprobsStep && T >= 2048)) p.waves = 1;
  else if (p.splits == 1 && T < kLongFew && V >= 16 * kLogprobsStep) p.waves = 16;
  return p;
}

// Parts that a workspace for T rows holds.  (Rows times splits never pass
// kParts + T - 1 with T < kFull, nor T times the most splits: a bound that does
// not fall as T grows.)
inline int64_t logprobs_parts(int64_t T, int32_t V) {
  const int64_t most = logprobs_most_splits(V);
  if (most < 2) return 0;
  return T * most < 2 * kParts ? T * most : 2 * kParts;
}

}  // namespace bnn
