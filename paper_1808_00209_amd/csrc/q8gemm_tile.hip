// 8-bit matrix product of many rows whose operands lie on 16-byte steps
// (bnn_q8gemm) on the int8 matrix cores.
//
// A workgroup of WM x WN waves computes 32 TM WM rows x 32 TN WN outputs, a wave
// 32 TM x 32 TN.  128 bytes of every row of both operands (a stage) go from
// memory straight into LDS, S stages in turn: while one is multiplied the next
// ones are on their way.  A wave reads the operands of its next matrix
// instructions while the present ones run, also over the stages' ends: the wait
// and the barrier come before a stage's last products.
//
// LDS is filled in the order of the lanes, so rows are 128 bytes apart there;
// a row's eight 16-byte chunks are stored in an order of its own (chunk j at
// j ^ (row / 2 % 8), by the address each lane loads from), so that a wave's
// reads of one chunk from 32 rows spread over the banks.
//
// 8192 x 16384 outputs, K 4096, bf16 out: 488-509 us from card to card, 2.16 to
// 2.25e15 operations a second, what a large library product of these bytes
// reaches here (2.24e15); the card's clock is at 1.7 GHz then, the matrix cores
// busy in 60 % of the cycles.  Tried there: four waves of 128 x 128 (half the
// LDS reads; 488 us against 490), bands of 2 to 16 row tiles (497-506).  Outputs
// stored by each lane as they came took 640 us: through LDS they leave in runs.
// 256 x 4096 outputs, K 4096 (a tile of 64 per CU): 10 us, 3.3 of start and end
// and 0.18-0.2 per stage of 16 KB, 38 bytes a cycle into the CU's LDS (the wait
// for a stage's loads is counted, so that two later stages stay on their way:
// 17.8 us without).  Tried there: K split over the waves (10.6), stages of 256
// bytes (11.1), six stages (10.9).
#include "q8gemm.hpp"

namespace bnn {
namespace {

constexpr int kBK = 128;
constexpr int kChunks = kBK / 16;
constexpr int kSteps = kBK / 32;  // matrix instructions along a stage

__device__ __forceinline__ int place(int row, int j) { return row * kChunks + (j ^ ((row >> 1) & 7)); }

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

__device__ const v4i q8_zeros[1] = {{0, 0, 0, 0}};

// Workgroups per CU: as many as its 160 KB of LDS hold, up to two, but one where
// a wave's sums fill 128 registers.
constexpr int per_cu(int TM, int TN, int WM, int WN, int S) {
  const int lds = S * 32 * (WM * TM + WN * TN) * kBK;
  return TM * TN < 8 && 2 * lds <= 160 * 1024 ? 2 : 1;
}

template <class T, int TM, int TN, int WM, int WN, int S>
__global__ __launch_bounds__(64 * WM * WN, WM * WN / 4 * per_cu(TM, TN, WM, WN, S)) void q8_tile_kernel(
    Q8Args a, int cols, int tiles, int per_xcd, int band) {
  constexpr int kNT = 64 * WM * WN;
  constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN, kRows = BM + BN;
  constexpr int kLoads = kRows * kChunks / kNT;  // of a thread, per stage
  __shared__ v4i lds[S][kRows * kChunks];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, c = lane & 31;
  // Workgroups go to the 8 XCDs in turn: each XCD has a run of tiles of its own,
  // in bands of `band` row tiles, so that what its L2 holds is used by many.
  const int idx = static_cast<int>(blockIdx.x & 7) * per_xcd + static_cast<int>(blockIdx.x >> 3);
  if (static_cast<int>(blockIdx.x >> 3) >= per_xcd || idx >= tiles) return;
  const int row_tiles = tiles / cols;
  const int b = idx / (band * cols), in = idx - b * band * cols;
  const int high = min(band, row_tiles - b * band);
  const int64_t m0 = static_cast<int64_t>(b * band + in % high) * BM;
  const int n0 = in / high * BN;

  // Thread i of a stage's load l fills LDS slot l * kNT + i: chunk
  // (slot % 8) ^ (row / 2 % 8) of row slot / 8.
  const int8_t* src[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int slot = l * kNT + tid, row = slot / kChunks;
    const int j = (slot & 7) ^ ((row >> 1) & 7);
    const int8_t* p = row < BM ? a.x + min(m0 + row, a.M - 1) * a.x_stride
                               : a.w + static_cast<int64_t>(min(n0 + row - BM, a.N - 1)) * a.w_stride;
    src[l] = p + 16 * j;
  }
  const int stages = (a.K + kBK - 1) / kBK;
  const int whole = a.K / kBK;  // stages that K fills
  // Load l of stage `it`.
  auto fetch = [&](int it, int st, int l) {
    __builtin_amdgcn_global_load_lds((global_void*)(src[l] + it * kBK),
                                     (lds_void*)(&lds[st][l * kNT + wave * 64]), 16, 0, 0);
  };
  // Before the short stage is fetched: a chunk that would pass the row's end is
  // loaded from elsewhere, x's from zeros, w's from its row's start.
  auto redirect = [&]() {
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int slot = l * kNT + tid, row = slot / kChunks;
      const int j = (slot & 7) ^ ((row >> 1) & 7);
      if (whole * kBK + 16 * j + 16 > a.K)
        src[l] = (row < BM ? reinterpret_cast<const int8_t*>(q8_zeros) : src[l] - 16 * j) - whole * kBK;
    }
  };
  // K not of whole chunks: a row's last bytes, as the end of the 16 before the
  // row's end (x's that belong to the chunk before: 0), which the short stage's
  // chunk of both operands holds once the loads are there.
  const bool ragged = a.K % 16 != 0;
  constexpr int kEnds = (kRows + kNT - 1) / kNT;
  v4i ends[kEnds] = {};
  if (ragged) {
#pragma unroll
    for (int l = 0; l < kEnds; ++l) {
      const int row = l * kNT + tid;
      if (row < BM)
        ends[l] = low_bytes_cleared(
            *reinterpret_cast<const v4i_any*>(a.x + min(m0 + row, a.M - 1) * a.x_stride + a.K - 16),
            16 - a.K % 16);
      else if (row < kRows)
        ends[l] = *reinterpret_cast<const v4i_any*>(
            a.w + static_cast<int64_t>(min(n0 + row - BM, a.N - 1)) * a.w_stride + a.K - 16);
    }
  }
  auto write_ends = [&](int st) {
#pragma unroll
    for (int l = 0; l < kEnds; ++l) {
      const int row = l * kNT + tid;
      if (row < kRows) lds[st][place(row, a.K % kBK / 16)] = ends[l];
    }
    __syncthreads();
  };

  v16i acc[TM][TN] = {};
  constexpr int MF = TM * TN, OP = TM + TN;
  const int wm = wave / WN * 32 * TM, wn = wave % WN * 32 * TN;
  // A step's operands (rows of x, then of w) are read one step ahead, or with
  // few products per step, which are done before a read is, one stage ahead.
  constexpr bool kStageAhead = MF <= 2;
  constexpr int kSlots = kStageAhead ? 2 * kSteps : 2;
  static_assert(!kStageAhead || S % 2 == 0, "a stage's registers are its buffer's");
  v4i op[kSlots][OP];
  auto read = [&](int to, int st, int s, int o) {
    const int row = o < TM ? wm + 32 * o + c : BM + wn + 32 * (o - TM) + c;
    op[to][o] = lds[st][place(row, 2 * s + h)];
  };
  // its rows' and outputs' factors, used behind the products
  float xs[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i)
    xs[i] = a.x_scale ? a.x_scale[min(m0 + wm + 32 * i + c, a.M - 1)] : 1.0f;
  const int own = min(n0 + wn + lane, a.N - 1);
  const float ws = a.w_scale ? a.w_scale[own] : 1.0f;
  const float bias = a.bias ? a.bias[own] : 0.0f;

  // Loads that go straight to LDS count as loads from memory: a barrier alone says
  // nothing about them, so their wait stands here, before it.
  auto meet_all = [&]() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  constexpr int kAhead = kStageAhead ? S : S - 1;  // stages on their way at a stage's start
#pragma unroll
  for (int st = 0; st < kAhead; ++st) {
    if (st >= stages) break;
    if (st == whole) redirect();
#pragma unroll
    for (int l = 0; l < kLoads; ++l) fetch(st, st, l);
  }
  meet_all();
  if (ragged && whole == 0) write_ends(0);
#pragma unroll
  for (int s = 0; s < (kStageAhead ? kSteps : 1); ++s)
#pragma unroll
    for (int o = 0; o < OP; ++o) read(s, 0, s, o);
  // The next stage is there, for all waves, and nobody reads the one before.
  // With kAhead stages on their way, all but the newest S - 2 have come.
  auto meet = [&](bool counted) {
    if (counted && S > 2)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * kLoads) : "memory");
    else
      meet_all();
  };
  // Stage `it`, in buffer st.  Main: stage it + kAhead is a whole one, and
  // fetched between the products.
  auto stage = [&](int it, int st, auto main) {
    constexpr bool kMain = decltype(main)::value;
    const bool more = kMain || it + kAhead < stages;
    auto fetch_rest = [&]() {
      if (!kMain && more) {
        if (it + kAhead == whole) redirect();
#pragma unroll
        for (int l = 0; l < kLoads; ++l) fetch(it + kAhead, (st + kAhead) % S, l);
      }
    };
    auto next = [&]() {
      meet(more);
      if (!kMain && ragged && it + 1 == whole) {
        __syncthreads();
        write_ends((st + 1) % S);
      }
    };
    if constexpr (kStageAhead) next();
    fetch_rest();
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const bool last = s == kSteps - 1;
      const int from = last && !kStageAhead ? MF / 2 : 0;  // reads stand behind products [from, MF)
#pragma unroll
      for (int m = 0; m < MF; ++m) {
        if (!kStageAhead && last && m == from) next();
        const int now = kStageAhead ? (st & 1) * kSteps + s : s & 1;
        const int i = m / TN, j = m % TN;
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(op[now][TM + j], op[now][i], acc[i][j], 0, 0, 0);
        if (m >= from) {
#pragma unroll
          for (int o = (m - from) * OP / (MF - from); o < (m - from + 1) * OP / (MF - from); ++o) {
            if (kStageAhead) read(((st + 1) & 1) * kSteps + s, (st + 1) % S, s, o);
            else if (last) read((s + 1) & 1, (st + 1) % S, 0, o);
            else read((s + 1) & 1, st, s + 1, o);
          }
        }
        constexpr int kOver = 2 * MF;  // the loads stand behind the first products
        if (kMain && s * MF + m < kOver) {
#pragma unroll
          for (int l = (s * MF + m) * kLoads / kOver; l < (s * MF + m + 1) * kLoads / kOver; ++l)
            fetch(it + kAhead, (st + kAhead) % S, l);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  int it = 0;
  for (; it + S - 1 + kAhead < whole; it += S) {
#pragma unroll
    for (int st = 0; st < S; ++st) stage(it + st, st, std::true_type{});
  }
  for (; it < stages; it += S) {
#pragma unroll
    for (int st = 0; st < S; ++st) {
      if (it + st >= stages) break;
      stage(it + st, st, std::false_type{});
    }
  }

  __syncthreads();  // (the operands' last reads)

  // Outputs.  Register e of lane (h, c) is output 8 (e / 4) + 4 h + e % 4 of row
  // c: four neighbours at a time go to LDS (a region per wave), 32 rows x 32 TN
  // outputs, and from there to memory in whole runs of a row.
  constexpr int kCols = 32 * TN;
  constexpr int kRowBytes = kCols * static_cast<int>(sizeof(T)) + 16;
  constexpr int kRegion = 2 * kCols * 4 + 32 * kRowBytes;
  static_assert(kNT / 64 * kRegion <= static_cast<int>(sizeof(lds)), "the outputs' regions fit");
  static_assert(kRegion % 16 == 0, "aligned regions");
  char* mine = reinterpret_cast<char*>(&lds[0][0]) + wave * kRegion;
  float* factors = reinterpret_cast<float*>(mine);  // w_scale, then bias
  char* out = mine + 2 * kCols * 4;
  if (lane < kCols) {
    factors[lane] = ws;
    factors[kCols + lane] = bias;
  }
  T* y = static_cast<T*>(a.y);
  constexpr int kVec = 16 / sizeof(T), kPerRow = kCols / kVec;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = 32 * j + 8 * g + 4 * h;
        T v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = q8_output<T>(acc[i][j][4 * g + e], xs[i], factors[n + e], factors[kCols + n + e]);
        __builtin_memcpy(__builtin_assume_aligned(out + c * kRowBytes + n * sizeof(T), 4 * sizeof(T)), v,
                         sizeof(v));
      }
#pragma unroll
    for (int q = lane; q < 32 * kPerRow; q += 64) {
      const int row = q / kPerRow, n = n0 + wn + q % kPerRow * kVec;
      const int64_t m = m0 + wm + 32 * i + row;
      const v4i v = *reinterpret_cast<const v4i*>(out + row * kRowBytes + q % kPerRow * 16);
      if (m >= a.M || n >= a.N) continue;
      T* at = y + m * a.N + n;
      if (n + kVec <= a.N) {
        *reinterpret_cast<v4i_any*>(at) = v;
      } else {
        T part[kVec];
        __builtin_memcpy(part, &v, 16);
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (n + e < a.N) at[e] = part[e];
      }
    }
  }
}

template <int TM, int TN, int WM, int WN, int S>
void launch_shape(const Q8Args& a, hipStream_t s) {
  constexpr int BM = 32 * WM * TM, BN = 32 * WN * TN;
  const int64_t cols = (a.N + BN - 1) / BN, rows = (a.M + BM - 1) / BM;
  const int tiles = static_cast<int>(rows * cols);  // M * N <= 2^35: below 2^24
  const int per_xcd = (tiles + 7) / 8;
  const int band = 8;
  with_real_type(a.dtype, [&](auto t) {
    q8_tile_kernel<decltype(t), TM, TN, WM, WN, S>
        <<<8 * per_xcd, 64 * WM * WN, 0, s>>>(a, static_cast<int>(cols), tiles, per_xcd, band);
  });
}

}  // namespace

hipError_t launch_q8_tile(const Q8Args& a, Q8Form form, hipStream_t s) {
  switch (form) {
    case kQ8Tile256: launch_shape<4, 2, 2, 4, 2>(a, s); break;
    case kQ8Pair128: launch_shape<2, 2, 2, 2, 2>(a, s); break;
    case kQ8Tile128: launch_shape<2, 1, 2, 4, 4>(a, s); break;
    default: launch_shape<1, 1, 2, 2, 4>(a, s); break;
  }
  return hipGetLastError();
}

}  // namespace bnn
