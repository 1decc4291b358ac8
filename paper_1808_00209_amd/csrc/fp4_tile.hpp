// The main loop of a binary GEMM tile on the fp4 matrix cores, for kernels
// whose data rows may lie anywhere: a workgroup of 4 waves computes up to 256
// outputs x 128 rows, a wave 64 outputs x 32 PT rows.  Per k-step two weight
// operands (expanded in registers from packed words) and PT data operands
// serve 2 PT MFMAs.  The data rows are staged in LDS, expanded once per
// workgroup, 256 bits of each at a time in two buffers: while one chunk's
// MFMAs run, the next one's words (loaded a chunk earlier) are expanded into
// the other, a few vector instructions after each MFMA (up to 4 hide behind
// it), and one barrier separates the chunks.  Words and bits past K are staged
// as fp4 0.0, so their products vanish whatever the weight words hold there.
#pragma once

#include <type_traits>

#include "fp32_split.hpp"
#include "fp4_expand.hpp"
#include "kernels.hpp"

namespace bnn {

constexpr int kTileNT = 256;             // threads of a workgroup
constexpr int kTileKS = 4;               // k-steps (64 bits) per chunk
constexpr int kTilePS = 2 * kTileKS + 1; // LDS entries per staged row (odd: no conflicts)
constexpr int kTileRows = 128;           // data rows per block, at most (staged, used or not)
constexpr size_t kTileLds = size_t{2} * kTileRows * kTilePS * 16;
constexpr int kTileRsrcWord3 = 0x00020000;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, static_cast<int>(bytes),
                                           kTileRsrcWord3);
}

__device__ __forceinline__ v4i tile_load4(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
  return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
}

// What a wave needs to run the loop.  Lane half h feeds words 4 h .. 4 h + 3
// of a chunk in both operands, one 16-byte load per row and half.
struct TileLoop {
  __amdgpu_buffer_rsrc_t ra, rb;  // data rows and weight rows
  uint32_t woff[2];  // byte offsets of weight rows f0 + c and f0 + 32 + c, + 16 h
  int32_t K, Kw;     // bits and words of a row
  int32_t chunks;    // of 8 words
  uint32_t tmask;    // valid bits of word Kw - 1
  int32_t wpi;       // the wave's place along the rows
};

// acc[tf][pt] += the 32 x 32 sums of outputs f0 + 32 tf and rows
// 32 (wpi PT + pt) .. (register e of lane (h, c): output 8 (e / 4) + 4 h +
// e % 4, row c).  Every thread of the workgroup takes part.  row_off() is the
// byte offset of row tid / 2 of the block's 128 in ra, + 16 (tid % 2): called
// after the first weight loads, which need not wait for what it reads.
template <int PT, class RowOff>
__device__ __forceinline__ void tile_loop(v16f (&acc)[2][PT], v4i* act, const TileLoop& t,
                                          RowOff&& row_off) {
  constexpr int kRing = PT == 4 ? 2 : 4;  // chunks of words in flight
  constexpr int buf1 = kTileRows * kTilePS;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, c = lane & 31;
  const uint32_t smask = __builtin_amdgcn_readfirstlane(0x88888888u);
  uint32_t vfill;
  asm("v_mov_b32 %0, 0x22222222" : "=v"(vfill));
  const uint32_t tmask = t.tmask;
  const int nch = t.chunks;
  const int whole = t.K >> 8;  // chunks of 256 valid bits
  const int sdst = (tid >> 1) * kTilePS + 4 * (tid & 1);

  // Word s of the thread's half of chunk ch, expanded into LDS.  MASK: the
  // chunk may hold words or bits past K (or lie past it altogether).
  auto stage_word = [&](const v4i& x, int ch, int s, int buf, auto mc) {
    const uint32_t w = static_cast<uint32_t>(x[s]);
    v4i e;
    if constexpr (!decltype(mc)::value) {
      e[0] = static_cast<int>(and_or(w << 3, smask, vfill));
      e[1] = static_cast<int>(and_or(w << 2, smask, vfill));
      e[2] = static_cast<int>(and_or(w << 1, smask, vfill));
      e[3] = static_cast<int>(and_or(w, smask, vfill));
    } else {
      const int wi = 8 * ch + 4 * (tid & 1) + s;
      const uint32_t vm = wi < t.Kw - 1 ? ~0u : (wi == t.Kw - 1 ? tmask : 0u);
      const v8i p = expand_fp4(w & vm, smask, 0u), q = expand_fp4(vm, smask, 0u);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        e[r] = static_cast<int>(static_cast<uint32_t>(p[r]) | (static_cast<uint32_t>(q[r]) >> 2));
    }
    act[buf + sdst + s] = e;
  };

  v4i xr[kRing], wr[kRing][2];  // words of the next kRing chunks, in flight
  uint32_t aoff;
  auto load_x = [&](int r, int ch) {
    xr[r] = tile_load4(t.ra, aoff, static_cast<uint32_t>(ch) * 32);
  };
  auto load_w = [&](int r, int ch) {
#pragma unroll
    for (int tf = 0; tf < 2; ++tf)
      wr[r][tf] = tile_load4(t.rb, t.woff[tf], static_cast<uint32_t>(ch) * 32);
  };
#pragma unroll
  for (int r = 0; r < kRing; ++r) load_w(r, min(r, nch - 1));
  __builtin_amdgcn_sched_barrier(0);
  aoff = row_off();
#pragma unroll
  for (int r = 0; r < kRing; ++r) load_x(r, min(r, nch - 1));
  int abase[PT];
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) abase[pt] = ((t.wpi * PT + pt) * 32 + c) * kTilePS + 4 * h;
  if (whole > 0) {
#pragma unroll
    for (int s = 0; s < kTileKS; ++s) stage_word(xr[0], 0, s, 0, std::false_type{});
  } else {
#pragma unroll
    for (int s = 0; s < kTileKS; ++s) stage_word(xr[0], 0, s, 0, std::true_type{});
  }
  load_x(0, min(kRing, nch - 1));
  __syncthreads();

  // Data operands: with few row tiles a k-step is shorter than an LDS read
  // takes, so a whole chunk's are read at its start; with four, each is read
  // again as soon as both output tiles have used it.
  constexpr int NB = PT == 4 ? 1 : kTileKS;
  v4i B[NB][PT], A[2][2];  // A: [ring][output tile]
  auto expand_op = [&](v4i (&x)[2], int w, int tf, int k) {
    const uint32_t u = static_cast<uint32_t>(w);
    x[tf][k] = static_cast<int>(and_or(k == 3 ? u : u << (3 - k), smask, vfill));
  };
#pragma unroll
  for (int o = 0; o < 8; ++o) expand_op(A[0], wr[0][o / 4][0], o / 4, o % 4);

  // Chunk ch (ring slot r) from LDS buffer `buf`; stages chunk ch + 1 (its
  // words in the next slot) into `obuf`, loads the words of kRing chunks on.
  auto chunk = [&](int ch, auto rc, int buf, int obuf, auto mc) {
    constexpr int r = decltype(rc)::value;
    constexpr int r1 = (r + 1) % kRing;
#pragma unroll
    for (int s = 0; s < NB; ++s)
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) B[s][pt] = act[buf + abase[pt] + s];
#pragma unroll
    for (int s = 0; s < kTileKS; ++s) {
      const int ring = s & 1;
      const int rn = s + 1 < kTileKS ? r : r1, sn = s + 1 < kTileKS ? s + 1 : 0;
      if (s == kTileKS - 1) load_w(r, min(ch + kRing, nch - 1));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 2 * PT; ++m) {
        const int pt = m / 2, tf = m % 2;
        const v4i x = A[ring][tf], b = B[s % NB][pt];
        acc[tf][pt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}, v8i{b[0], b[1], b[2], b[3], 0, 0, 0, 0},
            acc[tf][pt], 4, 4, 0, 127, 0, 127);
#pragma unroll
        for (int o = m * 8 / (2 * PT); o < (m + 1) * 8 / (2 * PT); ++o)
          expand_op(A[ring ^ 1], wr[rn][o / 4][sn], o / 4, o % 4);
        if (NB == 1 && tf == 1 && s + 1 < kTileKS) B[0][pt] = act[buf + abase[pt] + s + 1];
        __builtin_amdgcn_sched_barrier(0);
      }
      stage_word(xr[r1], ch + 1, s, obuf, mc);
    }
    load_x(r1, min(ch + 1 + kRing, nch - 1));
    __syncthreads();
    // (a masked chunk may be the last: its products stay before that branch
    // instead of being moved past it, operands and all, into registers that
    // spill)
    if constexpr (decltype(mc)::value) {
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) asm volatile("" : "+v"(acc[0][pt]), "+v"(acc[1][pt]));
    }
  };
  // (kRing chunks per trip: LDS buffers and ring slots keep fixed names)
  auto trip = [&](int ch, auto mc) {
    constexpr bool mask = decltype(mc)::value;
    chunk(ch, std::integral_constant<int, 0>{}, 0, buf1, mc);
    if (mask && ch + 1 >= nch) return;
    chunk(ch + 1, std::integral_constant<int, 1>{}, buf1, 0, mc);
    if constexpr (kRing == 4) {
      if (mask && ch + 2 >= nch) return;
      chunk(ch + 2, std::integral_constant<int, 2 % kRing>{}, 0, buf1, mc);
      if (mask && ch + 3 >= nch) return;
      chunk(ch + 3, std::integral_constant<int, 3 % kRing>{}, buf1, 0, mc);
    }
  };
  int ch = 0;
  // (with K in whole chunks nothing is masked: what the last chunk stages is
  // read by no one)
  const int plain = whole == nch ? nch - kRing : whole - kRing - 1;
  for (; ch <= plain; ch += kRing) trip(ch, std::false_type{});
  for (; ch < nch; ch += kRing) trip(ch, std::true_type{});
}

// Starts the sums of an output at v in all 32 rows (lane c of half 0 holds output
// c's value, the other half 0): one bf16 MFMA per tile, where clearing its
// registers takes 16 instructions; A an output's value as three bf16 parts
// (exact: half-integers below 2^23), B ones.
template <int PT>
__device__ __forceinline__ void tile_start(v16f (&acc)[PT], float v) {
  const uint16_t ones[8] = {kBf16One, kBf16One, kBf16One, kBf16One,
                            kBf16One, kBf16One, kBf16One, kBf16One};
  v4i b = __builtin_bit_cast(v4i, bf16x8(ones));
  const Split3 sp = split3(v);
  const uint16_t parts[8] = {bf16_bits(sp.p0), bf16_bits(sp.p1), bf16_bits(sp.p2), kBf16Zero,
                             kBf16Zero, kBf16Zero, kBf16Zero, kBf16Zero};
#pragma unroll
  for (int pt = 0; pt < PT; ++pt) {
    asm volatile("" : "+v"(b));  // (else one product and 16 PT moves)
    acc[pt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16x8(parts), __builtin_bit_cast(v8bf, b),
                                                      v16f{}, 0, 0, 0);
  }
}

}  // namespace bnn
