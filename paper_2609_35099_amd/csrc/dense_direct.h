// Large bfloat16 products: operands straight from memory to LDS.
#pragma once
#include "dense_tile.h"

namespace {

// One operand's way.  A wave's load instruction fills 1 KB of LDS in order, lane by
// lane: the exchange of slots (Plane) is made by choosing what each lane reads.
template <Form F, int R, int BK, int WAVES>
struct Feed {
  static constexpr int N = R * BK * 2 / 1024 / WAVES;  // instructions of a wave and step
  using Lds = Plane<F, R, BK, 1, true>;
  const char* base;  // of the next step
  int64_t step;      // bytes
  unsigned off[N];   // of the lane's pieces
  int at;            // values of LDS before the wave's first
  // rows: output indexes (kPaired: of a half)
  __device__ __forceinline__ Feed(const Side& s, int64_t r0, int64_t rows, int64_t k0) {
    const int l = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
    at = wave * N * 512;
    base = static_cast<const char*>(s.p) + 2 * (F == kAlong ? r0 * s.ld + k0 : k0 * s.ld + r0);
    step = 2 * (F == kAlong ? (int64_t)BK : BK * s.ld);
    constexpr int S = Lds::S, PER = kWave / S;  // slots of an LDS row, LDS rows of an instruction
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (wave * N + i) * PER + l / S, slot = (Lds::off(row, l % S) - row * Lds::W) / 8;
      if constexpr (F == kAlong) {
        const int last = rows - r0 < R ? (int)(rows - r0) - 1 : R - 1;
        off[i] = 2u * (unsigned)(imin(row, last) * (int)s.ld + slot * 8);
      } else {
        // pieces past the columns' end read the last one: their results are not stored
        const int left = rows - r0 < R ? (int)(rows - r0) - 8 : R;
        const int half = F == kPaired && slot / 4 % 2 ? (int)rows : 0;
        const int col = F == kPaired ? slot / 8 * 32 + slot % 4 * 8 : slot * 8;
        off[i] = 2u * (unsigned)(row * (int)s.ld + half + imin(col, left));
      }
    }
  }
  // A half of the next step's loads (0, then 1).  In asm, so that the compiler, which cannot tell the buffers'
  // loads apart across the loop, does not wait for all of them at the first read;
  // DirectTile waits.  Nothing is loaded to registers; m0 is set before each use, here and
  // by the compiler.
  __device__ __forceinline__ void next(Lds& to, int half) {
    typedef __attribute__((address_space(3))) unsigned short* lds;
    const unsigned first = (unsigned)(uintptr_t)(lds)&to.v[0][at];
#pragma unroll
    for (int i = half * N / 2; i < (half + 1) * N / 2; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(first + i * 1024), "v"(off[i]),
                   "s"(base)
                   : "memory");
    if (half) base += step;
  }
};

// A tile of 256 x 256 by eight waves of 128 x 64, steps of 64 in two buffers: the
// loads of a step are in flight while the one before it is multiplied, and none of
// them passes through registers.  Whole pieces of 16 aligned bytes only
// (direct_side), reductions in multiples of 64.  Sums run over the reduction in the
// order of the other tiles: the same bits.
// The loads are issued in two halves behind the first reads of LDS, which they would
// hold up: 16,384 x 1,024 by 4,096 columns of reduction takes 135 us so, 144 with all
// of them first, 150 with all of them behind the first reads (the library 95).
// Other tiles, measured with the loads first: a product of 8,192 x 4,096 x 8,192 in a
// gated layer took 465 us (the library's bare one 409); tiles of 256 x 128 by four
// waves, two to a CU, steps of 32 in three buffers 578; steps of 32 in four buffers
// 478; four waves of 128 x 128 643, and 540 with the next fragments read beside the
// products; the two waves of a SIMD in turns, one's products beside the other's reads,
// 490; steps of 32 in five buffers with the next fragments read beside the products
// 500.  Of the 16,384 x 1,024 the products alone took 105 us, the loads alone 74.
template <Form FA, Form FB>
struct DirectTile {
  static constexpr int BM = 256, BN = 256, BK = 64, WM = 2, WN = 4, THREADS = WM * WN * kWave;
  static constexpr int RM = BM / WM / 32, RN = BN / WN / 32;
  using A = Feed<FA, BM, BK, WM * WN>;
  using B = Feed<FB, BN, BK, WM * WN>;
  static_assert(RN == 2);
  struct Buf {
    typename A::Lds a;
    typename B::Lds b;
  };
  f16v acc[RM][RN];

  // Where the wave's part of the tile begins.
  static __device__ __forceinline__ int row0() { return uniform(threadIdx.x / kWave) / WN * (32 * RM); }
  static __device__ __forceinline__ int col0() { return uniform(threadIdx.x / kWave) % WN * (32 * RN); }
  // between(i): after the reads of the i-th 16 indexes, before their products
  template <class Fn>
  __device__ __forceinline__ void multiply(const Buf& s, Fn&& between) {
#pragma unroll
    for (int k = 0; k < BK; k += 16) {
      bf8v x[RM], y[RN];
#pragma unroll
      for (int j = 0; j < RN; ++j) y[j] = s.b.frag(0, col0() + 32 * j, k);
#pragma unroll
      for (int i = 0; i < RM; ++i) x[i] = s.a.frag(0, row0() + 32 * i, k);
      between(k / 16);
#pragma unroll
      for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[j], x[i], acc[i][j], 0, 0, 0);
    }
  }
  // Sums over reduction indexes [k0, end), a multiple of BK, of the tile at (r0, c0).
  __device__ __forceinline__ void run(Buf& s0, Buf& s1, const Side& sa, const Side& sb, int64_t r0, int64_t rows, int c0,
                                      int cols, int64_t k0, int64_t end) {
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    A fa(sa, r0, rows, k0);
    B fb(sb, c0, cols, k0);
    const int n = (int)((end - k0) / BK);
    for (int h = 0; h < 2; ++h) fa.next(s0.a, h), fb.next(s0.b, h);
    // past the barrier every wave's loads are there, and every wave is done with the
    // buffer that is filled next
    auto step = [&](int s, Buf& now, Buf& next) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      multiply(now, [&](int i) {
        if (i < 2 && s + 1 < n) fa.next(next.a, i), fb.next(next.b, i);
      });
    };
    for (int s = 0; s < n; s += 2) {
      step(s, s0, s1);
      if (s + 1 < n) step(s + 1, s1, s0);
    }
  }
  // The wave's staging for its results, once all waves are here.
  static __device__ __forceinline__ float (*stage(Buf& s0, Buf& s1))[32 * RN + 4] {
    typedef float Stage[32][32 * RN + 4];
    constexpr int PER = WM * WN / 2;  // of a buffer
    static_assert(sizeof(Buf) >= PER * sizeof(Stage));
    const int w = uniform(threadIdx.x / kWave);
    __syncthreads();
    return reinterpret_cast<Stage*>(w < PER ? &s0 : &s1)[w % PER];
  }
};

// f(0) .. f(N - 1) with constants, so that indexed registers stay registers whatever
// the size of f.
template <class F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// Whether a side can be read that way: whole aligned pieces, offsets within a tile in
// 32 bits.  cols: of a memory row (or of each of its halves).
inline bool direct_side(const Side& s, int64_t cols) {
  return s.p && (reinterpret_cast<uintptr_t>(s.p) & 15u) == 0 && s.ld % 8 == 0 && cols % 8 == 0 && s.ld <= 1 << 21;
}

}  // namespace
