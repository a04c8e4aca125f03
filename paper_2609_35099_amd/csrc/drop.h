// Masks of dropout, made from a counter where they are used and never stored.
#pragma once
#include "layers.h"

namespace {

// Random bits: Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", 2011), a keyed bijection of 128-bit counters.
// The key is the seed, the counter (row mod 2^32, row / 2^32 2^17 + column / 8,
// offset), so that a value's bits depend on nothing but the seed, the offset, its
// row and its column: not on strides, types, launch shapes or the columns beside it.
// A call gives eight columns 16 bits each.  Bits of 32 would cost twice the
// multiplications, which a read and a write of bfloat16 do not hide; with 16, p is
// rounded to a multiple of 2^-16, and what is kept grows by the rounded one.
struct Drop {
  const int64_t* counter;  // added to the offset when the kernel runs (null: 0)
  uint64_t seed, offset;
  unsigned t;              // dropped where the bits are below it; 0: nothing is
  float grow;
};
inline bool good_drop(double p, const int64_t* counter) {
  return p >= 0.0 && p <= 1.0 && !(reinterpret_cast<uintptr_t>(counter) & 7u);
}
inline Drop drop_of(double p, uint64_t seed, uint64_t offset, const int64_t* counter) {
  Drop d{counter, seed, offset, (unsigned)std::nearbyint(p * 65536.0), 0.0f};
  if (d.t < 65536) d.grow = (float)(65536.0 / (65536 - d.t));
  return d;
}

struct Dropper {
  unsigned k0, k1, c2, c3, t;
  __device__ __forceinline__ Dropper(const Drop& d) {
    uint64_t o = d.offset;
    if (d.t && d.counter) o += (uint64_t)*d.counter;
    k0 = (unsigned)d.seed, k1 = (unsigned)(d.seed >> 32), c2 = (unsigned)o, c3 = (unsigned)(o >> 32), t = d.t;
  }
  // Which of the V values from column col (a multiple of V) on are kept, a bit each.
  template <int V>
  __device__ __forceinline__ unsigned kept(int64_t row, int col) const {
    static_assert(V == 4 || V == 8);
    unsigned w[4] = {(unsigned)row, (unsigned)(row >> 32) << 17 | (unsigned)col >> 3, c2, c3}, a = k0, b = k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t p = (uint64_t)w[0] * 0xD2511F53u, q = (uint64_t)w[2] * 0xCD9E8D57u;
      w[0] = (unsigned)(q >> 32) ^ w[1] ^ a;
      w[1] = (unsigned)q;
      w[2] = (unsigned)(p >> 32) ^ w[3] ^ b;
      w[3] = (unsigned)p;
      a += 0x9E3779B9u, b += 0xBB67AE85u;
    }
    if constexpr (V == 4) {
      if (col & 4) w[0] = w[2], w[1] = w[3];
    }
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      m |= (w[i] & 0xffffu) >= t ? 1u << (2 * i) : 0u;
      m |= w[i] >> 16 >= t ? 2u << (2 * i) : 0u;
    }
    return m;
  }
};

}  // namespace
