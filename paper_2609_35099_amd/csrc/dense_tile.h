// The tile product behind the dense layers, on the bf16 matrix cores.
//
// A workgroup takes a BM x BN tile of the output; the reduction runs in steps of
// BK.  Per step the threads load both operands' pieces of 16 bytes into
// registers (the next step's are in flight during the instructions) and write
// them to LDS as bf16; waves read fragments for v_mfma_f32_32x32x16_bf16, in
// which lane l holds row (or column) l % 32 at reduction indexes 8 (l / 32) on.
//
// An operand lies in memory either with its reduction contiguous (kAlong: x of
// the forward, dz and W of dx) or with its rows or columns contiguous (kAcross:
// W of the forward, x and dz of dW).  LDS keeps the order of memory, so global
// loads and LDS writes are whole pieces either way: fragments of the first come
// by 16-byte reads, of the second by ds_read_b64_tr_b16, where 16 lanes read
// four rows of 16 values and receive a column each.
//
// float32 operands are split into three bf16 terms of 8 bits each with their
// signs, h + m + l = x exactly, in three planes; a product is the six term
// products down to 2^-24 of it (hl, lh, mm, hm, mh, hh, added smallest first in
// one chain).  The bf16 units run 16 times as fast as the float32 ones, so six
// products on them beat one there.  Terms are scaled by 2^24, so that none of a
// normal operand is subnormal (the instruction takes those as zero), and sums
// scaled back; a sum that is not finite then (an infinity or a NaN among the
// operands, an operand past 2e31, a sum past 1e24) is computed again from memory
// in float32.  8-bit operands are exact in one term: three products.
#pragma once
#include "layers.h"

namespace {

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));

enum Form { kAlong, kAcross };

constexpr float kTermScale = 0x1p24f, kTermBack = 0x1p-48f;

__device__ __forceinline__ unsigned pack2(float a, float b) {
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f2v{a, b}, bf2v));
}
// The terms of a and b, packed; a and b become what the terms so far leave.
__device__ __forceinline__ unsigned term2(float& a, float& b) {
  const unsigned t = pack2(a, b);
  a -= __uint_as_float(t << 16), b -= __uint_as_float(t & 0xffff0000u);
  return t;
}

// One operand of a tile product, or the pre-activation beside it.
struct Side {
  const void* p;      // full: memory rows (kAlong: of an output index, kAcross: of a reduction index) at p + i ld
  int64_t ld;
  const int8_t* q;    // packed (p null): ld values and ldc exponents a row
  const uint8_t* c;
  int64_t ldc;
  int64_t total;      // values from the first to the last, at least a piece
};

// LDS planes of R rows (or columns) by BK reduction indexes.  16-byte slots are
// exchanged so that the lanes of one pass of a read cover all banks: along, by
// the row's number among those that share the banks; across, the pairs of slots
// of the four rows that one transposing read takes.
template <Form F, int R, int BK, int P>
struct Plane {
  static constexpr int W = F == kAlong ? BK : R;          // values of an LDS row
  static constexpr int S = W / 8;                         // slots of one
  static constexpr int kShare = F == kAlong ? (S >= 16 ? 1 : 16 / S) : 1;  // rows over all banks
  unsigned short v[P][R * BK];
  static __device__ __forceinline__ int off(int row, int slot) {
    const int x = F == kAlong ? (row / kShare) & (S - 1 < 15 ? S - 1 : 15) : (2 * (row & 3)) & (S - 1);
    return row * W + ((slot ^ x) * 8);
  }
  // The fragment of rows (columns) r0 + l % 32 at reduction indexes k0 + 8 (l / 32) on.
  __device__ __forceinline__ bf8v frag(int p, int r0, int k0) const {
    const int l = threadIdx.x % kWave;
    if constexpr (F == kAlong) {
      return *reinterpret_cast<const bf8v*>(&v[p][off(r0 + l % 32, k0 / 8 + l / 32)]);
    } else {
      typedef __attribute__((address_space(3))) s4v* lds;
      const int k = k0 + 8 * (l / 32) + (l % 16) / 4, col = r0 + 16 * ((l / 16) % 2) + 4 * (l % 4);
      union {
        s4v h[2];
        bf8v f;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(&v[p][off(k, col / 8) + col % 8]));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(&v[p][off(k + 4, col / 8) + col % 8]));
      return u.f;
    }
  }
};

// A thread's N pieces of V values of a tile of memory rows of W values, as they
// lie in memory; R and BK are the tile's output and reduction indexes.
template <class T, Form F, int R, int BK, int THREADS, bool Q>
struct Fetch {
  static constexpr int V = Elem<T>::V, W = F == kAlong ? BK : R, PER = W / V, N = R * BK / V / THREADS;
  static constexpr int BITS = Q ? 8 : 8 * sizeof(T);      // of a value
  static_assert(N * V * THREADS == R * BK && THREADS % PER == 0);
  using E = typename std::conditional<Q, int8_t, T>::type;
  using Raw = typename std::conditional<Q, typename std::conditional<V == 4, unsigned, u2v>::type, u4v>::type;
  typedef Raw Any __attribute__((aligned(sizeof(E))));
  Raw raw[N];
  unsigned char exps[Q ? N : 1];
  Cutting cut[N];  // of pieces that are not whole

  static __device__ __forceinline__ int row_of(int i) { return threadIdx.x / PER + i * (THREADS / PER); }
  static __device__ __forceinline__ int col_of() { return threadIdx.x % PER * V; }
  // The reduction index before which the tile's pieces are inside the matrix's
  // span: where rows or columns end within the tile (across), pieces past the end
  // hold values of the next row, which only reach results that are not stored.
  static __device__ __forceinline__ int64_t whole_until(const Side& s, int64_t r0, int64_t rows) {
    constexpr int64_t all = (int64_t)1 << 62;
    if (F == kAlong || r0 + W <= rows) return all;
    const int64_t room = s.total - r0 - W;
    int64_t m = room < 0 ? 0 : room / s.ld + 1;
    if constexpr (Q) {
      const int64_t left = s.total / s.ld * s.ldc - r0 / kGroup - W / kGroup, mc = left < 0 ? 0 : left / s.ldc + 1;
      m = mc < m ? mc : m;
    }
    return m;
  }

  // The tile at output index r0 and reduction index k0 of an operand with `rows`
  // output indexes; reduction indexes from `end` on are zero; output indexes
  // past the end read as the last row (along) or zero (across): their results
  // are not stored.  WHOLE: all reduction indexes and all pieces are inside (up to
  // whole_until(); a loop of its own: with both ways in one, the loaded registers
  // were copied where the ways meet, which waits for the loads).
  // Otherwise pieces may reach into the next row (ld_span) and are cut when they
  // are used.
  template <bool WHOLE>
  __device__ __forceinline__ void load(const Side& s, int64_t r0, int64_t rows, int64_t k0, int64_t end) {
    // memory row m0 + row_of(i), column c0 + col_of(): the uniform part in the base
    const int64_t m0 = F == kAlong ? r0 : k0, c0 = F == kAlong ? k0 : r0;
    const int64_t mend = F == kAlong ? rows : end, cend = F == kAlong ? end : rows;
    const E* p = (Q ? reinterpret_cast<const E*>(s.q) : static_cast<const E*>(s.p)) + (m0 * s.ld + c0);
    const uint8_t* pc = Q ? s.c + (m0 * s.ldc + c0 / kGroup) : nullptr;
    const int mlast = mend - m0 < 1024 ? (int)(mend - m0) - 1 : 1023;
    const int lc = col_of();
    if constexpr (WHOLE) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t m = F == kAlong ? imin(row_of(i), mlast) : row_of(i);
        raw[i] = *reinterpret_cast<const Any*>(p + (m * s.ld + lc));
        if constexpr (Q) exps[i] = pc[m * s.ldc + lc / kGroup];
      }
      return;
    }
    const E* first = Q ? reinterpret_cast<const E*>(s.q) : static_cast<const E*>(s.p);
    const int left = cend - c0 < 1024 ? (int)(cend - c0) : 1024;  // columns from c0 on, at least one
    const int n = left - lc < V ? (left - lc > 0 ? left - lc : 0) : V;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool in = F == kAlong || row_of(i) <= mlast;
      const int64_t m = imin(row_of(i), mlast);
      raw[i] = ld_span<Raw>(first, (m0 + m) * s.ld + c0 + lc, s.total, in ? n : 0, cut[i]);
      if constexpr (Q) exps[i] = pc[m * s.ldc + imin(lc, left - 1) / kGroup];
    }
  }
  // Piece i as it lies in memory, and its values.
  template <bool WHOLE>
  __device__ __forceinline__ Raw bits(int i) const {
    return WHOLE ? raw[i] : cut[i](raw[i]);
  }
  template <bool WHOLE>
  __device__ __forceinline__ void get(int i, float (&v)[V]) const {
    const Raw b = bits<WHOLE>(i);
    if constexpr (Q) {
      Raw8<V> r;
      // a step's exponent only where something was read: a NaN step times a zero is NaN
      r.e = !WHOLE && cut[i].none() ? 0u : exps[i];
      if constexpr (V == 4) r.w[0] = b; else r.w[0] = b.x, r.w[1] = b.y;
      get8(r, v);
    } else {
      Elem<T>::get(__builtin_bit_cast(typename Elem<T>::vec, b), v);
    }
  }
};

// What an operand is: as it is, packed, or dy act'(z) from dy and z in full or
// packed (the last two never exist in memory).  In bfloat16 they are rounded here
// to its 8 bits, as operands of the instruction: dx and dW are then off by 2.4e-3 of
// their size, of which their own rounding at the end is 1.7e-3.  Sixteen bits, as two
// terms, would leave the latter alone and double the instructions of both products
// (290 us of a training step of 640 at 16,384 x 1,024 x 4,096).
enum Kind { kFull, kPacked, kGradFull, kGradPacked };

// One operand's way from memory to LDS.
template <class T, Form F, int R, int BK, int THREADS, Kind KD>
struct Loader {
  static constexpr int V = Elem<T>::V;
  static constexpr bool Q = KD == kPacked, G = KD >= kGradFull;
  static constexpr int P = sizeof(T) == 2 || Q ? 1 : 3;   // planes
  using Lds = Plane<F, R, BK, P>;
  using Main = Fetch<T, F, R, BK, THREADS, Q>;
  using Pre = Fetch<T, F, R, BK, THREADS, KD == kGradPacked>;
  static constexpr int N = Main::N;
  struct None {};
  Main x;
  typename std::conditional<G, Pre, None>::type z;

  static __device__ __forceinline__ int64_t whole_until(const Side& s, const Side& pre, int64_t r0, int64_t rows) {
    const int64_t m = Main::whole_until(s, r0, rows);
    if constexpr (!G) return m;
    const int64_t p = Pre::whole_until(pre, r0, rows);
    return p < m ? p : m;
  }
  template <bool WHOLE>
  __device__ __forceinline__ void load(const Side& s, const Side& pre, int64_t r0, int64_t rows, int64_t k0,
                                       int64_t end) {
    x.template load<WHOLE>(s, r0, rows, k0, end);
    if constexpr (G) z.template load<WHOLE>(pre, r0, rows, k0, end);
  }
  // To LDS; `sum` (where wanted) grows by the values of the thread's columns.
  template <bool SUM, bool WHOLE>
  __device__ __forceinline__ void store(Lds& l, int act, float (&sum)[V]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = Main::row_of(i), col = Main::col_of();
      const int o = Lds::off(row, col / 8) + col % 8;
      if constexpr (KD == kFull && sizeof(T) == 2 && !SUM) {
        *reinterpret_cast<u4v*>(&l.v[0][o]) = x.template bits<WHOLE>(i);
      } else {
        float v[V];
        x.template get<WHOLE>(i, v);
        if constexpr (G) {
          float w[V];
          z.template get<WHOLE>(i, w);
          act_grad_piece(act, w, v);
        }
        if constexpr (SUM)
#pragma unroll
          for (int e = 0; e < V; ++e) sum[e] += v[e];
        if constexpr (P == 1) {
          // packed values are exact; those of float32 tiles are scaled
          unsigned b[V / 2];
#pragma unroll
          for (int e = 0; e < V / 2; ++e)
            b[e] = sizeof(T) == 4 ? pack2(v[2 * e] * kTermScale, v[2 * e + 1] * kTermScale) : pack2(v[2 * e], v[2 * e + 1]);
          if constexpr (V == 4) *reinterpret_cast<u2v*>(&l.v[0][o]) = u2v{b[0], b[1]};
          else *reinterpret_cast<u4v*>(&l.v[0][o]) = u4v{b[0], b[1], b[2], b[3]};
        } else {
          float a = v[0] * kTermScale, b = v[1] * kTermScale, c = v[2] * kTermScale, d = v[3] * kTermScale;
#pragma unroll
          for (int t = 0; t < 3; ++t) {
            const unsigned x = term2(a, b), y = term2(c, d);
            *reinterpret_cast<u2v*>(&l.v[t][o]) = u2v{x, y};
          }
        }
      }
    }
  }
};

// The tile and its reduction.  WM x WN waves; acc[i][j]: rows 32 i on and
// columns 32 j on of the wave's part; the columns take the instruction's A side,
// so that a lane holds row l % 32 and columns 8 (e / 4) + 4 (l / 32) + e % 4.
template <class T, Form FA, Form FB, int BM, int BN, int BK, int WM, int WN, Kind KA, Kind KB, bool SUM, int BUFS>
struct Tile {
  static constexpr int THREADS = WM * WN * kWave, TM = BM / WM, TN = BN / WN, RM = TM / 32, RN = TN / 32;
  using LA = Loader<T, FA, BM, BK, THREADS, KA>;
  using LB = Loader<T, FB, BN, BK, THREADS, KB>;
  union Shared {
    struct {
      typename LA::Lds a;
      typename LB::Lds b;
    } in[BUFS];
    float out[WM * WN][32][TN + 4];
    float sums[SUM ? THREADS / LB::Main::PER : 1][SUM ? BN : 1];
  };
  f16v acc[RM][RN];
  float sum[LB::V];  // SUM: of this thread's columns of B

  __device__ __forceinline__ void step(const typename LA::Lds& a, const typename LB::Lds& b, int row0, int col0) {
    constexpr int PA = LA::P, PB = LB::P;
#pragma unroll
    for (int k = 0; k < BK; k += 16) {
      bf8v x[PA][RM], y[PB][RN];
#pragma unroll
      for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int i = 0; i < RM; ++i) x[p][i] = a.frag(p, row0 + 32 * i, k);
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int j = 0; j < RN; ++j) y[p][j] = b.frag(p, col0 + 32 * j, k);
      // pairs of terms, smallest products first
#pragma unroll
      for (int s = PA + PB - 2 < 2 ? PA + PB - 2 : 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < PA; ++p) {
          const int q = s - p;
          if (q < 0 || q >= PB) continue;
#pragma unroll
          for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[q][j], x[p][i], acc[i][j], 0, 0, 0);
        }
      if constexpr (RM * RN > 4) __builtin_amdgcn_sched_barrier(0);
    }
  }

  struct Args {
    Side a, b, z;      // z: beside the operand that is a gradient
    int act;
  };
  // Sums over reduction indexes [k0, end) of the tile at (r0, c0) of rows x cols
  // (ONLY: the column sums of B alone).
  template <bool ONLY>
  __device__ __forceinline__ void run(Shared& sh, const Args& g, int64_t r0, int64_t rows, int c0,
                                      int cols, int64_t k0, int64_t end) {
    const int w = uniform(threadIdx.x / kWave), row0 = w / WN * TM, col0 = w % WN * TN;
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    if constexpr (SUM)
#pragma unroll
      for (int e = 0; e < LB::V; ++e) sum[e] = 0.0f;
    int64_t until = ONLY ? end : LA::whole_until(g.a, g.z, r0, rows);
    const int64_t ub = LB::whole_until(g.b, g.z, c0, cols);
    until = until < ub ? until : ub;
    until = until < end ? until : end;
    const int64_t whole = until > k0 ? k0 + (until - k0) / BK * BK : k0;
    steps<true, ONLY>(sh, g, r0, rows, c0, cols, k0, whole, row0, col0);
    steps<false, ONLY>(sh, g, r0, rows, c0, cols, whole, end, row0, col0);
  }
  template <bool WHOLE, bool ONLY>
  __device__ __forceinline__ void steps(Shared& sh, const Args& g, int64_t r0, int64_t rows, int c0, int cols, int64_t k,
                                        int64_t end, int row0, int col0) {
    if (k >= end) return;
    LA la;
    LB lb;
    auto load = [&](int64_t at) {
      if constexpr (!ONLY) la.template load<WHOLE>(g.a, g.z, r0, rows, at, end);
      lb.template load<WHOLE>(g.b, g.z, c0, cols, at, end);
    };
    auto store = [&](int buf) {
      float none[LA::V];
      if constexpr (!ONLY) la.template store<false, WHOLE>(sh.in[buf].a, g.act, none);
      lb.template store<SUM, WHOLE>(sh.in[buf].b, g.act, sum);
    };
    load(k);
    __syncthreads();
    int cur = 0;
    if constexpr (BUFS == 2) store(0);
    for (; k < end; k += BK) {
      if constexpr (BUFS == 1) store(0);
      __syncthreads();
      const bool more = k + BK < end;
      if (more) load(k + BK);
      if constexpr (!ONLY) step(sh.in[cur].a, sh.in[cur].b, row0, col0);
      if constexpr (BUFS == 1) {
        __syncthreads();
      } else {
        if (more) store(cur ^ 1);
        cur ^= 1;
      }
    }
  }
  // The column sums of B over the tile's reduction, f(col, value), col within the
  // tile: the threads of a column in order.
  template <class Fn>
  __device__ __forceinline__ void finish_sums(Shared& sh, Fn&& f) {
    using M = typename LB::Main;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < LB::V; ++e) sh.sums[threadIdx.x / M::PER][M::col_of() + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < BN) {
      float v = 0.0f;
#pragma unroll
      for (int r = 0; r < THREADS / M::PER; ++r) v += sh.sums[r][threadIdx.x];
      f((int)threadIdx.x, v);
    }
  }

  // The wave's rows in blocks of 32 to out(row, col, results) with row and col of
  // the block within the tile; every wave's staging is its own.
  template <class Fn>
  __device__ __forceinline__ void finish(Shared& sh, Fn&& out) {
    const int w = uniform(threadIdx.x / kWave), row0 = w / WN * TM, col0 = w % WN * TN;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RM; ++i) out(row0 + 32 * i, col0, sh.out[w], acc[i]);
  }
};

// The results of 32 rows and 32 RN columns go through a wave's own staging, so
// that a lane gets pieces of V values of a row (row l / PER of every PASS rows,
// columns V (l % PER) on) and rows are written whole.
template <class T, int RN>
struct Rows32 {
  static constexpr int V = Elem<T>::V, TN = 32 * RN, PER = TN / V, PASS = kWave / PER, N = 32 / PASS, PITCH = TN + 4;
  static_assert(kWave % PER == 0 && 32 % PASS == 0);
  static constexpr float kBack = sizeof(T) == 2 ? 1.0f : kTermBack;
  static __device__ __forceinline__ int row() { return threadIdx.x % kWave / PER; }
  static __device__ __forceinline__ int col() { return threadIdx.x % PER * V; }
  static __device__ __forceinline__ void put(float (*out)[PITCH], const f16v (&acc)[RN]) {
    const int l = threadIdx.x % kWave;
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < RN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f4v*>(&out[l % 32][32 * j + 8 * g + 4 * (l / 32)]) =
            f4v{acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]} * kBack;
    wait();
  }
  // The wave's own writes: LDS serves a wave's accesses in order.
  static __device__ __forceinline__ void wait() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
  // Piece i of the lane.
  static __device__ __forceinline__ void get(const float (*out)[PITCH], int i, float (&v)[V]) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const f4v t = *reinterpret_cast<const f4v*>(&out[i * PASS + row()][col() + e]);
      v[e] = t.x, v[e + 1] = t.y, v[e + 2] = t.z, v[e + 3] = t.w;
    }
  }
  // Whether a sum of the wave is not finite.
  static __device__ __forceinline__ bool bad(const f16v (&acc)[RN]) {
    float z = 0.0f;
#pragma unroll
    for (int j = 0; j < RN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) z = fmaf(acc[j][e], 0.0f, z);
    return __ballot(z != 0.0f) != 0;
  }
  // Replaces the sums that are not finite by again(row, col).
  template <class Fn>
  static __device__ __forceinline__ void mend(float (*out)[PITCH], Fn&& again) {
#pragma clang loop unroll(disable)
    for (int i = 0; i < 32 * TN; i += kWave) {
      const int at = i + threadIdx.x % kWave, r = at / TN, c = at % TN;
      const float v = out[r][c];
      if (v * 0.0f != 0.0f) out[r][c] = again(r, c);
    }
    wait();
  }
};

}  // namespace
