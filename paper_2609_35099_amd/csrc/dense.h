// Dense layers, shared by their units: arguments, the epilogue, the tile kernel
// and how a product is cut.
#pragma once
#include "dense_direct.h"

// A backward call, checked.
struct DenseBwdCall {
  e3_dtype dtype;
  const void *x, *W, *z, *dy;
  const int8_t *xq, *zq;
  const uint8_t *xc, *zc;
  void *dx, *dW, *db;
  char* ws;
  int64_t ldx, ldz, lddy, lddx, M, K, N;
  int act;
  hipStream_t st;
  bool given;  // dy is a finished dz, db is not wanted: ws has no room for either
};
e3_status dense_bwd_f32(const DenseBwdCall& c);
e3_status dense_bwd_bf16(const DenseBwdCall& c);

struct DenseArgs {
  Side a, b, pre;  // rows of A by columns of B over the reduction; the z of one that is a gradient
  int grad_act;
  int64_t rows, red;
  int cols;
  int64_t chunk;  // reduction indexes per split
  int splits;
  float* part;    // partial sums [splits][rows cols + tail], instead of the epilogue
  int64_t pitch;  // of a split's
  void* sums;     // column sums of B (one split; else after each split's partial sums)
  // epilogue
  const void *bias, *res;
  void *y, *z;
  int8_t *zq, *yq;
  uint8_t *zc, *yc;
  int64_t ldr, ldy, ldz;
  int act;
  bool nt;  // y (and z) streams
};
// bfloat16 products with operands straight to LDS, in a unit of their own
// (dense_direct.hip): x W, dz W^T and x^T dz.
e3_status dense_direct_fwd(const DenseArgs& a, hipStream_t st);
e3_status dense_direct_dx(const DenseArgs& a, hipStream_t st);
e3_status dense_direct_dw(const DenseArgs& a, hipStream_t st);

namespace {

// What follows the sums of one piece of a row, row0 + lr with row0 uniform (so
// that a thread multiplies by a row stride once, not per piece).  The lanes of a
// group of 32 columns take part together, also where rows (ok) or columns end.
// The piece of the bias is loaded once for all rows, that of the residual ahead
// of the sums.
template <class T>
struct Tail {
  static constexpr int V = Elem<T>::V;
  float bias[V];
  __device__ __forceinline__ Tail(const DenseArgs& a, int col) {
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = 0.0f;
    if (a.bias) ld_piece<T>(static_cast<const T*>(a.bias) + col, a.cols - col, bias);
  }
  struct Raw {
    u4v v;
    Cutting cut;
  };
  static constexpr unsigned kUncut = 128;
  static __device__ __forceinline__ Raw residual(const DenseArgs& a, int64_t row0, int lr, bool ok, int col) {
    Raw r{{}, {kUncut}};
    if (!a.res) return r;
    const int64_t total = (a.rows - 1) * a.ldr + a.cols;
    const int n = a.cols - col;
    const T* p = static_cast<const T*>(a.res);
    if (total >= V)
      r.v = ld_span<u4v>(p, (ok ? row0 + lr : 0) * a.ldr + col, total, !ok || n < 0 ? 0 : n < V ? n : V, r.cut);
    else
      r.v = __builtin_bit_cast(u4v, ld_raw<T>(p + (row0 * a.ldr + (lr * a.ldr + col)), ok ? n : 0));
    return r;
  }
  // FAST: the piece is inside the row, y streams, and there is neither a residual
  // nor an output beside it (plain()), so that a round of a loop over rows has no
  // branch around a load or store: the loads that the next round waits for are
  // older than the stores, and only a known number of stores lets the wait leave
  // them in flight.
  // BARE: there is no residual.
  template <bool FAST = false, bool BARE = FAST>
  __device__ __forceinline__ void out(const DenseArgs& a, int64_t row0, int lr, bool ok, int col, Raw res,
                                      float (&v)[V]) const {
    const int n = FAST ? V : ok ? a.cols - col : 0;
    auto at = [&](int64_t ld) { return row0 * ld + (lr * ld + col); };
    auto pack = [&](int8_t* q, uint8_t* c) {
      const int64_t groups = (a.cols + kGroup - 1) / kGroup;
      pack8_piece<V>(v, col, n, q + (row0 * a.cols + (int64_t)lr * a.cols), c + (row0 * groups + lr * groups));
    };
    if (FAST || a.bias)
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += bias[i];
    if (!FAST && a.z) st_piece<T>(static_cast<T*>(a.z) + at(a.ldz), n, v, a.nt);
    if (!FAST && a.zq) pack(a.zq, a.zc);
    act_piece(a.act, v);
    if (!BARE && a.res) {
      float u[V];
      if (__ballot(res.cut.down_keep != kUncut)) res.v = res.cut(res.v);
      Elem<T>::get(__builtin_bit_cast(typename Elem<T>::vec, res.v), u);
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += u[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = Elem<T>::round(v[i]);
    if constexpr (FAST) __builtin_nontemporal_store(Elem<T>::put(v), reinterpret_cast<typename Elem<T>::vec*>(static_cast<T*>(a.y) + at(a.ldy)));
    else st_piece<T>(static_cast<T*>(a.y) + at(a.ldy), n, v, a.nt);
    if (!FAST && a.yq) pack(a.yq, a.yc);
  }
  static bool plain(const DenseArgs& a) { return a.nt && !a.res && !a.z && !a.zq && !a.yq; }
};
template <class T, int V>
__device__ __forceinline__ void dense_tail(const DenseArgs& a, int64_t row0, int lr, bool ok, int col, float (&v)[V]) {
  const Tail<T> tail(a, col);
  tail.out(a, row0, lr, ok, col, Tail<T>::residual(a, row0, lr, ok, col), v);
}

// Value (m, c) of a memory row m of a tile's operand.
template <class T, Kind KD>
__device__ __forceinline__ float side_value(const Side& s, const Side& pre, int act, int64_t m, int64_t c) {
  auto packed = [&](const Side& p) { return (float)p.q[m * p.ld + c] * step8(p.c[m * p.ldc + c / kGroup]); };
  auto full = [&](const Side& p) { return Elem<T>::one(static_cast<const T*>(p.p)[m * p.ld + c]); };
  if constexpr (KD == kPacked) return packed(s);
  if constexpr (KD == kGradFull) return full(s) * act_grad(act, full(pre));
  if constexpr (KD == kGradPacked) return full(s) * act_grad(act, packed(pre));
  return full(s);
}
// A sum again from memory, in float32.
template <class T, Form FA, Form FB, Kind KA, Kind KB>
__device__ __forceinline__ float dense_again(const DenseArgs& a, int64_t row, int col, int64_t k0, int64_t end) {
  float sum = 0.0f;
#pragma clang loop unroll(disable)
  for (int64_t k = k0; k < end; ++k) {
    const float u = side_value<T, KA>(a.a, a.pre, a.grad_act, FA == kAlong ? row : k, FA == kAlong ? k : row);
    const float w = side_value<T, KB>(a.b, a.pre, a.grad_act, FB == kAlong ? col : k, FB == kAlong ? k : col);
    sum = fmaf(u, w, sum);
  }
  return sum;
}

// What a tile kernel is, apart from its size.
template <class T_, Form FA_, Form FB_, Kind KA_, Kind KB_, bool SUM_>
struct Job {
  using T = T_;
  static constexpr Form FA = FA_, FB = FB_;
  static constexpr Kind KA = KA_, KB = KB_;
  static constexpr bool SUM = SUM_;  // with the column sums of B
};
// The results of rows row0 to row0 + 31 and 32 RN columns from col0 on.  BARE: neither
// residual nor partial sums.
template <class J, int RN, bool FAST = false, bool BARE = FAST>
__device__ __forceinline__ void rows32_out(const DenseArgs& a, const Tail<typename J::T>& tail, int split, int64_t row0,
                                           int col0, int64_t k0, int64_t end, float (*out)[32 * RN + 4],
                                           const f16v (&acc)[RN]) {
  using T = typename J::T;
  using R = Rows32<T, RN>;
  constexpr int V = R::V;
  const int col = col0 + R::col(), lr = R::row();
  typename Tail<T>::Raw res[R::N];
#pragma unroll
  for (int i = 0; i < R::N; ++i)
    if (!BARE) res[i] = Tail<T>::residual(a, row0 + i * R::PASS, lr, row0 + i * R::PASS + lr < a.rows, col);
  R::put(out, acc);
  if constexpr (sizeof(T) == 4) {
    if (R::bad(acc))
      R::mend(out, [&](int r, int c) {
        return row0 + r < a.rows && col0 + c < a.cols
                   ? dense_again<T, J::FA, J::FB, J::KA, J::KB>(a, row0 + r, col0 + c, k0, end)
                   : 0.0f;
      });
  }
#pragma unroll
  for (int i = 0; i < R::N; ++i) {
    const int64_t rowu = row0 + i * R::PASS;
    const bool ok = FAST || rowu + lr < a.rows;
    float v[V];
    R::get(out, i, v);
    if (!BARE && a.part) {
      float* p = a.part + (split * a.pitch + rowu * a.cols) + ((int64_t)lr * a.cols + col);
#pragma unroll
      for (int e = 0; e < V; e += 4)
        st_piece<float>(p + e, (ok ? a.cols - col : 0) - e, reinterpret_cast<float(&)[4]>(v[e]));
    } else {
      tail.template out<FAST, BARE>(a, rowu, lr, ok, col, res[i], v);
    }
  }
  __builtin_amdgcn_wave_barrier();
}
template <class J, int RN, bool FAST = false>
__device__ __forceinline__ void rows32_out(const DenseArgs& a, int split, int64_t row0, int col0, int64_t k0, int64_t end,
                                           float (*out)[32 * RN + 4], const f16v (&acc)[RN]) {
  const Tail<typename J::T> tail(a, col0 + Rows32<typename J::T, RN>::col());
  rows32_out<J, RN, FAST>(a, tail, split, row0, col0, k0, end, out, acc);
}

// Tiles by type and size, with us per call in turn with the other side.
//   bfloat16, 256 x 256 (where DirectTile cannot read the operands, or the reduction is
//     short): 16 waves of 64 x 64, steps of 32, two buffers, one workgroup per CU:
//     16,384 x 1,024 x 4,096 dx 142, dW 149 (the library's products 100, 166).  The
//     forward takes 256 x 128 by 8 waves, two workgroups per CU, so
//     that one's activations run beside the other's product: 164 for the bare product
//     (155 with 256 x 256, the library's 132), but with gelu 185 (187), and a training
//     step with z in 8 bits 656 (670).
//   bfloat16, 128 and 64: 4 waves, steps of 64, two buffers, two workgroups and
//     more.  (The sizes above by them: forward 190, backward 366 against 330.)
//   float32: one buffer of the three planes.  Rows along the reduction take 64 x
//     128 by 4 waves, four workgroups per CU that load, split and multiply beside
//     each other.  128 x 128 by 8 waves, two per CU, are slower where the reduction is
//     short (forward 100,000 x 128 x 256 64 against 85, 60,000 x 100 x 1,000 155
//     against 186, backward of 100,003 x 128 x 256 from 8 bits 138 against 167), as
//     fast at 16,384 x 1,024 x 1,024 (221, 223) and faster where it is long (4,096 x
//     2,048 x 1,024 124 against 116, 2,048 x 4,096 x 4,096 442 against 412; the
//     library 120 for the former).  Across, 128 x 128 by 4 waves (8 were 8% slower).
template <class J, int B>
struct TileOf {
  static constexpr bool f32 = sizeof(typename J::T) == 4, along = J::FA == kAlong, fwd = along && J::FB == kAcross;
  static constexpr int BM = f32 && along && B == 128 ? 64 : B, BN = B == 256 && fwd ? 128 : B;
  static constexpr int WM = B == 256 ? 4 : 2, WN = B == 256 ? BN / 64 : 2;
  static constexpr int BK = f32 || B == 256 ? 32 : 64, THREADS = WM * WN * kWave, OCC = B == 256 ? 4 : 2;
  using type = Tile<typename J::T, J::FA, J::FB, BM, BN, BK, WM, WN, J::KA, J::KB, J::SUM, f32 ? 1 : 2>;
};

// Which tile block u of tm x tn takes: blocks go round robin to the XCDs, so an
// XCD takes a contiguous eighth, eight row tiles by eight column tiles running
// together, which share their operands in its L2: bfloat16 40,000 x 515 x 1,021 100
// us against 108 in order, backward of 16,384 x 1,024 x 4,096 339 against 358, float32
// 16,384 x 1,024 x 1,024 232 against 239; 8,192 x 4,096 x 4,096 307 either way.
struct TileAt {
  int64_t m;
  int n;
};
__device__ __forceinline__ TileAt tile_at(int64_t u, int64_t tm, int tn) {
  const int64_t total = tm * tn, per = total / kXcd, extra = total % kXcd;
  if (total < 4 * kXcd || total >= (int64_t)1 << 31) return {u / tn, (int)(u % tn)};
  const unsigned x = (unsigned)(u % kXcd);
  const unsigned v = x * (unsigned)per + (x < extra ? x : (unsigned)extra) + (unsigned)(u / kXcd);
  const unsigned group = 8 * tn, g = v / group, w = v % group;
  const unsigned first = g * 8, size = tm - first < 8 ? (unsigned)(tm - first) : 8;
  return {first + w % size, (int)(w / size)};
}

// Tile number u of a product.
template <class J, class Tl, int BM, int BN, bool ONLY = false>
__device__ __forceinline__ void dense_block(const DenseArgs& a, typename Tl::Shared& sh, int64_t u) {
  using T = typename J::T;
  constexpr int V = Elem<T>::V;
  const int64_t tm = ONLY ? 1 : (a.rows + BM - 1) / BM;
  const int tn = (a.cols + BN - 1) / BN;
  if (u >= tm * tn * a.splits) return;
  const int split = (int)(u / (tm * tn));
  u -= split * (tm * tn);
  const TileAt at = tile_at(u, tm, tn);
  const int64_t r0 = at.m * BM;
  const int c0 = at.n * BN;
  const int64_t k0 = split * a.chunk, end = k0 + a.chunk < a.red ? k0 + a.chunk : a.red;
  Tl t;
  t.template run<ONLY>(sh, {a.a, a.b, a.pre, a.grad_act}, r0, a.rows, c0, a.cols, k0, end);
  if constexpr (J::SUM) {
    if (r0 == 0 && a.sums)
      t.finish_sums(sh, [&](int c, float v) {
        if (c0 + c >= a.cols) return;
        if (a.part) a.part[split * a.pitch + a.rows * a.cols + c0 + c] = v;
        else static_cast<T*>(a.sums)[c0 + c] = (T)v;
      });
  }
  if constexpr (!ONLY)
    t.finish(sh, [&](int r, int c, auto out, auto& acc) {
      rows32_out<J, Tl::RN>(a, split, r0 + r, c0 + c, k0, end, out, acc);
    });
}
template <class J, int B>
__global__ __launch_bounds__((TileOf<J, B>::THREADS), (TileOf<J, B>::OCC)) void k_dense(DenseArgs a) {
  using Tl = typename TileOf<J, B>::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  dense_block<J, Tl, TileOf<J, B>::BM, TileOf<J, B>::BN>(a, sh, block_id());
}
// Short reductions (up to 16 KK) over many rows: no LDS and no barriers before the
// epilogue.  A wave keeps the terms of its 32 NC columns of B in registers for
// good and walks row blocks of 32; lane l loads the eight values of row l % 32 at
// reduction indexes 16 kk + 8 (l / 32) on straight into the instruction's operand
// order, the next block's while it works on one.  The waves of a workgroup take
// neighbouring columns of the same rows.
// What bounds a short reduction is the write of y; tiles through LDS wait for
// their own loads, barriers and stores in turn.  156,000 x 64 x 1,664: bfloat16 113
// us (4.8 TB/s), float32 304 (tiles 421; bound by the vector unit, which splits
// every row once per wave); 1,248,000 x 64 x 64 59 (5.4 TB/s) and 131 (4.9).
template <class J, int KK, int NC, bool FAST>
__global__ __launch_bounds__(256, 2) void k_dense_panel(DenseArgs a) {
  using T = typename J::T;
  using R = Rows32<T, NC>;
  constexpr bool f32 = sizeof(T) == 4;
  constexpr int V = Elem<T>::V, P = f32 ? 3 : 1, Q = 8 / V;
  constexpr bool GF = J::KA == kGradFull, GP = J::KA == kGradPacked;
  static_assert(J::FA == kAlong && J::KA != kPacked && J::KB == kFull && !J::SUM);
  __shared__ __align__(16) float out[4][32][R::PITCH];
  const int l = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), K = (int)a.red;
  const int groups = (a.cols + 32 * NC - 1) / (32 * NC);
  const int64_t w = block_id() * 4 + wave;
  const int64_t chunk = w / groups;
  if (chunk >= a.splits) return;
  const int col0 = (int)(w % groups) * 32 * NC;
  const int h = 8 * (l / 32);
  // the wave's columns of B
  bf8v wf[P][KK][NC];
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = col0 + 32 * c + l % 32;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = 16 * k + h + e;
        const T* b = static_cast<const T*>(a.b.p);
        v[e] = at < K && col < a.cols ? Elem<T>::one(J::FB == kAlong ? b[col * a.b.ld + at] : b[at * a.b.ld + col]) : 0.0f;
        if (f32) v[e] *= kTermScale;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        u4v t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
        wf[p][k][c] = __builtin_bit_cast(bf8v, t);
      }
    }
  // a row block's values, as they lie in memory
  typename Elem<T>::vec x[KK][Q], zf[GF ? KK : 1][Q];
  Raw8<8> zp[GP ? KK : 1];
  const T* xp = static_cast<const T*>(a.a.p);
  const T* zfp = static_cast<const T*>(a.pre.p);
  auto load = [&](auto fast, int64_t block) {
    constexpr bool F = decltype(fast)::value;
    const int last = F ? 31 : a.rows - block * 32 < 32 ? (int)(a.rows - block * 32) - 1 : 31;
    const int64_t m = imin(l % 32, last);
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const int at = 16 * k + h;
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int n = F ? V : K - at - q * V;
        x[k][q] = ld_raw<T>(xp + block * 32 * a.a.ld + (m * a.a.ld + at + q * V), n);
        if constexpr (GF) zf[k][q] = ld_raw<T>(zfp + block * 32 * a.pre.ld + (m * a.pre.ld + at + q * V), n);
      }
      if constexpr (GP)
        zp[k] = ld_raw8<8>(a.pre.q + block * 32 * a.pre.ld + m * a.pre.ld,
                           a.pre.c + block * 32 * a.pre.ldc + m * a.pre.ldc, at, F ? 8 : K - at);
    }
  };
  bf8v xf[P][KK];
  auto terms = [&]() {
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      if constexpr (!f32 && !GF && !GP) {
        xf[0][k] = __builtin_bit_cast(bf8v, x[k][0]);
      } else {
        float v[8];
#pragma unroll
        for (int q = 0; q < Q; ++q) Elem<T>::get(x[k][q], reinterpret_cast<float(&)[V]>(v[q * V]));
        if constexpr (GF || GP) {
          float z[8];
          if constexpr (GP) {
            get8(zp[k], z);
          } else {
#pragma unroll
            for (int q = 0; q < Q; ++q) Elem<T>::get(zf[k][q], reinterpret_cast<float(&)[V]>(z[q * V]));
          }
          act_grad_piece(a.grad_act, z, v);
        }
        if constexpr (f32)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= kTermScale;
#pragma unroll
        for (int p = 0; p < P; ++p) {
          u4v t;
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
          xf[p][k] = __builtin_bit_cast(bf8v, t);
        }
      }
    }
  };
  auto product = [&](auto fast, int64_t block) {
    f16v acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int s = 2 * P - 2 < 2 ? 2 * P - 2 : 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int q = s - p;
          if (q < 0 || q >= P) continue;
#pragma unroll
          for (int c = 0; c < NC; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[q][k][c], xf[p][k], acc[c], 0, 0, 0);
        }
    rows32_out<J, NC, decltype(fast)::value>(a, 0, block * 32, col0, 0, a.red, out[wave], acc);
  };
  // FAST: whole row blocks by a loop without branches around loads and stores, and
  // what is left of the rows after it
  const int64_t blocks = FAST ? a.rows / 32 : (a.rows + 31) / 32;
  const std::integral_constant<bool, FAST> fast;
  if (chunk < blocks) {
    // a round ends with loads and begins with stores, so that its wait for the
    // loads of the one before leaves its own stores in flight; blocks past the
    // end load the last one again
    auto at = [&](int64_t b) { return b < blocks ? b : blocks - 1; };
    load(fast, chunk);
    terms();
    load(fast, at(chunk + a.splits));
    for (int64_t block = chunk; block < blocks; block += a.splits) {
      product(fast, block);
      terms();
      load(fast, at(block + 2 * (int64_t)a.splits));
    }
  }
  if (FAST && a.rows % 32 && chunk == blocks % a.splits) {
    load(std::false_type{}, blocks);
    terms();
    product(std::false_type{}, blocks);
  }
}
// The same where rows have columns for several waves: WPB waves of a workgroup
// bring each row block to LDS together, so that its terms are formed once and not
// by every wave (a third of the vector work in float32, which is what bounds the
// kernel above).  156,000 x 64 x 1,664 float32: 304 us there, 265 with 1,536 of the
// columns here (228) and the rest there; 156,000 x 32 x 1,664 190 us (5.6 TB/s), 194
// there.
// Two waves with a reduction of 64 are slower than none (421): LDS leaves six on a
// CU.  Columns are whole multiples of 64 WPB, the reduction is at most BK, y
// streams and is the only output.
template <class J, int BK, int WPB>
__global__ __launch_bounds__(WPB* kWave, 2) void k_dense_shared(DenseArgs a) {
  using T = typename J::T;
  using LA = Loader<T, kAlong, 32, BK, WPB * kWave, J::KA, false>;
  constexpr int NC = 2, KK = BK / 16, P = LA::P;
  static_assert(J::FA == kAlong && J::KA != kPacked && J::KB == kFull && !J::SUM);
  __shared__ __align__(16) typename LA::Lds in[2];
  __shared__ __align__(16) float out[WPB][32][Rows32<T, NC>::PITCH];
  const int l = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), K = (int)a.red;
  const int groups = a.cols / (64 * WPB);
  const int64_t chunk = block_id() / groups;
  if (chunk >= a.splits) return;
  const int col0 = ((int)(block_id() % groups) * WPB + wave) * 64;
  bf8v wf[P][KK][NC];
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = col0 + 32 * c + l % 32;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = 16 * k + 8 * (l / 32) + e;
        const T* b = static_cast<const T*>(a.b.p);
        v[e] = at < K ? Elem<T>::one(J::FB == kAlong ? b[col * a.b.ld + at] : b[at * a.b.ld + col]) : 0.0f;
        if (P > 1) v[e] *= kTermScale;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        u4v t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
        wf[p][k][c] = __builtin_bit_cast(bf8v, t);
      }
    }
  const int64_t blocks = (a.rows + 31) / 32, whole = a.rows / 32;
  LA la;
  float none[LA::V];
  auto load = [&](int64_t block) {
    if (block >= blocks) block = blocks - 1;
    // (the pieces of a short reduction are cut)
    if (K == BK) la.template load<true>(a.a, a.pre, block * 32, a.rows, 0, BK);
    else la.template load<false>(a.a, a.pre, block * 32, a.rows, 0, K);
  };
  int cur = 0;
  f16v acc[NC];
  auto product = [&]() {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      bf8v xf[P];
#pragma unroll
      for (int p = 0; p < P; ++p) xf[p] = in[cur].frag(p, 0, 16 * k);
#pragma unroll
      for (int s = 2 * P - 2 < 2 ? 2 * P - 2 : 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int q = s - p;
          if (q < 0 || q >= P) continue;
#pragma unroll
          for (int c = 0; c < NC; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[q][k][c], xf[p], acc[c], 0, 0, 0);
        }
    }
  };
  if (chunk >= blocks) return;  // the whole workgroup
  load(chunk);
  auto store = [&](typename LA::Lds& to) {
    if (K == BK) la.template store<false, true>(to, a.grad_act, none);
    else la.template store<false, false>(to, a.grad_act, none);
  };
  store(in[0]);
  load(chunk + a.splits);
  __syncthreads();
  int64_t block = chunk;
  for (; block < whole; block += a.splits) {
    product();
    store(in[cur ^ 1]);
    load(block + 2 * (int64_t)a.splits);
    rows32_out<J, NC, true>(a, 0, block * 32, col0, 0, a.red, out[wave], acc);
    __syncthreads();
    cur ^= 1;
  }
  if (block < blocks) {  // the last rows, fewer than 32
    product();
    rows32_out<J, NC>(a, 0, block * 32, col0, 0, a.red, out[wave], acc);
  }
}
// What a product's kernels are called in timings: by tile, and by row walk.
struct Names {
  const char *t64, *t128, *t256, *panel, *shared;
  const char* tile(int b) const { return b == 64 ? t64 : b == 128 ? t128 : t256; }
};
constexpr Names kNamesFwd{"dense_fwd_64", "dense_fwd_128", "dense_fwd_256", "dense_fwd_panel", "dense_fwd_shared"};
constexpr Names kNamesDx{"dense_bwd_dx_64", "dense_bwd_dx_128", "dense_bwd_dx_256", "dense_bwd_dx_panel",
                         "dense_bwd_dx_shared"};
constexpr Names kNamesDw{"dense_bwd_dw_64", "dense_bwd_dw_128", "dense_bwd_dw_256", nullptr, nullptr};
constexpr Names kNamesDb{"dense_bwd_db_64", "dense_bwd_db_128", "dense_bwd_db_256", nullptr, nullptr};
// Whether a product goes that way: a reduction that fits the registers beside its
// columns, and rows enough for the waves to walk.
template <class T>
constexpr int kPanel = sizeof(T) == 4 ? 64 : 128;
template <class T>
bool panel(int64_t rows, int64_t cols, int64_t red) {
  return red <= kPanel<T> && ((rows + 31) / 32) * ((cols + 63) / 64) >= 8192;
}
template <class J>
e3_status dense_panel(DenseArgs a, const Names& names, hipStream_t st) {
  using T = typename J::T;
  if constexpr (sizeof(T) == 4) {
    // Shared row blocks: four waves, or two where the terms of B are few (more
    // would leave them without registers for two workgroups per CU); the columns
    // past the last 256 in a launch of their own, which pays where there are many
    // before them, or where the kernel above would run its loop with branches and
    // they are not a few alone.  156,000 rows, in two launches against all above, us:
    // x 64 x 320 88 against 75, x 576 118 against 115, x 832 153 against 160, x 1,664
    // 266 against 304; x 40 x 300 109 against 89, x 320 84 against 88, x 640 127
    // against 158.
    const int64_t four = a.cols / 256 * 256, rest = a.cols - four;
    const bool two = four > 0 && (a.red % 16 == 0 && a.cols % 64 == 0 ? four >= 768 : rest >= 64);
    const int wpb = rest == 0 || (a.red > 32 && two) ? 4 : a.red <= 32 && a.cols % 128 == 0 ? 2 : 0;
    if (Tail<T>::plain(a) && wpb) {
      DenseArgs m = a;
      if (wpb == 4) m.cols = (int)four;
      const int64_t col = m.cols / (64 * wpb);
      m.splits = (int)std::min<int64_t>((a.rows + 31) / 32, std::max<int64_t>(1, 2048 / wpb / col));
      {
        TimedLaunch t_(names.shared, st);
        auto* k = wpb == 2 ? k_dense_shared<J, 32, 2> : a.red <= 32 ? k_dense_shared<J, 32, 4> : k_dense_shared<J, 64, 4>;
        hipLaunchKernelGGL(k, grid_of(m.splits * col), dim3(wpb * kWave), 0, st, m);
        E3_HIP(hipGetLastError());
      }
      if (m.cols == a.cols) return E3_OK;
      a.cols -= m.cols;
      a.b.p = static_cast<const T*>(a.b.p) + (J::FB == kAlong ? m.cols * a.b.ld : m.cols);
      a.y = static_cast<T*>(a.y) + m.cols;
      if (a.bias) a.bias = static_cast<const T*>(a.bias) + m.cols;
      return dense_panel<J>(a, names, st);
    }
  }
  // two workgroups per CU, each wave on row blocks of its own
  const int64_t groups = (a.cols + 63) / 64;
  a.splits = (int)std::min<int64_t>((a.rows + 31) / 32, std::max<int64_t>(1, 2048 / groups));
  const int64_t blocks = (a.splits * groups + 3) / 4;
  TimedLaunch t_(names.panel, st);
  auto go = [&](auto KK) {
    constexpr int kk = decltype(KK)::value;
    const bool fast = a.red == 16 * kk && a.cols % 64 == 0 && Tail<T>::plain(a);
    auto* k = fast ? k_dense_panel<J, kk, 2, true> : k_dense_panel<J, kk, 2, false>;
    hipLaunchKernelGGL(k, grid_of(blocks), dim3(256), 0, st, a);
  };
  if (a.red <= 32) go(std::integral_constant<int, 2>{});
  else if (sizeof(T) == 4 && a.red <= 48) go(std::integral_constant<int, 3>{});
  else if (a.red <= 64) go(std::integral_constant<int, 4>{});
  else if constexpr (sizeof(T) == 2) {
    if (a.red <= 96) go(std::integral_constant<int, 6>{});
    else go(std::integral_constant<int, 8>{});
  }
  E3_HIP(hipGetLastError());
  return E3_OK;
}

// The partial sums of the splits, in order, and the epilogue; after the last row
// the column sums beside them.
template <class T>
__global__ __launch_bounds__(256) void k_dense_join(DenseArgs a, int splits) {
  constexpr int V = Elem<T>::V;
  const int per = (a.cols + kGroup - 1) / kGroup * (kGroup / V);
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  const int col = (int)(i - row * per) * V;
  const int n = row < a.rows + (a.sums ? 1 : 0) ? a.cols - col : 0;
  float v[V] = {};
  const float* p = a.part + (row * a.cols + col);
  for (int s = 0; s < splits; s += 4) {
    float u[4][V];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < V; e += 4)
        ld_piece<float>(p + (s + j) * a.pitch + e, s + j < splits ? n - e : 0, reinterpret_cast<float(&)[4]>(u[j][e]));
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] += u[j][e];
  }
  if (row == a.rows && a.sums) {
    st_piece<T>(static_cast<T*>(a.sums) + col, n, v);
    return;  // whole groups: nothing is packed here
  }
  if (a.y) dense_tail<T, V>(a, row, 0, row < a.rows, col, v);
}

// ------------------------------------------------------------ host
// How a product is cut: square tiles, and splits of its reduction where the
// tiles alone would leave much of the card idle.
struct Cut {
  int tile, splits;  // TileOf's B
  int64_t tiles, chunk;
};
enum Product { kForward, kDx, kDw };
constexpr int kFill = 512;  // workgroups of the smaller tiles that fill the card
Cut dense_cut(e3_dtype t, int64_t rows, int64_t cols, int64_t red, Product which) {
  Cut c{};
  auto tiles = [&](int b, int bn = 0) {
    bn = bn ? bn : b;
    return ((rows + b - 1) / b) * ((cols + bn - 1) / bn);
  };
  const int64_t t128 = tiles(128), t256 = tiles(256);
  int64_t fill = kFill;
  // Small tiles where there are few: more of them are on a CU and wait for memory
  // together (bfloat16 4,096 x 512 x 1,024 14 us against 27, 2,048^3 36 against 39;
  // float32 4,096 x 512 x 1,024 38 against 41, but 2,048^3 125 against 107: long
  // reductions are split instead, as is dW of 100,003 x 128 x 256, 65 against 84).
  const bool few = t == E3_BF16 ? t128 < kFill && red < 8192 : t128 < kFill / 2 && red < 1024;
  c.tile = rows <= 64 || cols <= 64 || few ? 64 : 128;
  if (t == E3_BF16 && rows > 128 && cols > 128) {
    // rounds of the card by the time of one: four times the work of a 128 x 128
    // tile, of which two run on a CU at 0.78 of the rate; splits of 2,048 at least
    const int64_t s = std::max<int64_t>(1, std::min(256 / t256, red / 2048));
    const double big = (double)((t256 * s + 255) / 256) * 4.0 / (double)s;
    if (t256 * s >= 192 && big <= (double)((t128 + kFill - 1) / kFill) * 2.56)
      c.tile = 256, fill = which == kForward ? 512 : 256;
  }
  c.tiles = tiles(c.tile);
  if (c.tile == 256 && which == kForward) c.tiles = tiles(256, 128);
  if (c.tile == 128 && t == E3_F32 && which != kDw) c.tiles = tiles(64, 128), fill = 2 * kFill;  // 64 x 128 by TileOf
  // at least 256 indexes a split; few tiles of few indexes take down to 64
  int64_t least = c.tiles * (red / 256) < kFill / 8 ? 64 : c.tile == 256 ? 2048 : 256;
  // What a launch to join them takes is longer: bfloat16 300^3 8.8 us against 13.8, 64
  // x 384 x 512 8.9 against 13.5, float32 16 x 300 x 300 11.8 against 13.7, 100 x 384 x
  // 100 13.3 against 13.7, backward of 380 x 300 x 200 22 against 28.
  if (red <= 384) least = 384;
  const int64_t s = std::max<int64_t>(
      1, std::min<int64_t>({fill / std::max<int64_t>(c.tiles, 1), (red + least - 1) / least, 256}));
  c.chunk = std::max<int64_t>(64, ((red + s - 1) / s + 63) / 64 * 64);
  c.splits = (int)std::max<int64_t>(1, (red + c.chunk - 1) / c.chunk);
  return c;
}
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
// Partial sums of a cut product and of `tail` sums beside it.
size_t cut_bytes(const Cut& c, int64_t rows, int64_t cols, int64_t tail = 0) {
  return c.splits > 1 ? up256((size_t)c.splits * (rows * cols + tail) * sizeof(float)) : 0;
}
void set_cut(DenseArgs& a, const Cut& c, float* part, int64_t tail = 0) {
  a.chunk = c.chunk, a.splits = c.splits, a.part = c.splits > 1 ? part : nullptr, a.pitch = a.rows * a.cols + tail;
}

// Whether the products of the backward form dz from dy and z on the way to LDS:
// once per 128 columns of x, so for up to 256; wider layers write dz once.  Formed
// against written, silu, us: 60,003 x 64 x 256 float32 61 against 84, from 8 bits 56
// against 72; x 256 x 1,024 560 against 612, 484 against 521; bfloat16 x 64 x 256 36
// against 46, from 8 bits 38 against 45; x 256 x 256 82 against 86; x 256 x 1,024 201
// against 224.  bfloat16 from 8 bits past 128 columns unpacks, differentiates and
// rounds for every tile with too few registers for it in the largest: 60,003 x 256 x
// 256 155 against 83, x 1,024 549 against 208 (120,011 rows 1,688 against 351), and
// in the smaller ones 20,011 x 192 x 256 47 against 45, x 1,024 104 against 87; but
// few columns of dz cost little (45,011 x 192 x 64 45 against 51), and small layers
// save a launch (10,007 x 192 x 128 29 against 31, 3,000 x 200 x 300 22 against 29).
constexpr int64_t kOnTheFly = 256;
bool forms_dz(e3_dtype t, int64_t M, int64_t K, int64_t N, bool packed) {
  if (K > kOnTheFly) return false;
  if (!packed || t != E3_BF16 || K <= 128) return true;
  return (N <= 64 || M * N < (1 << 21)) && dense_cut(t, M, K, N, kDx).tile < 256;
}

struct DenseBwdWs {
  size_t dz, db, part, total;
  int64_t db_blocks, db_rows;
};
DenseBwdWs dense_bwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N, bool given = false) {
  const size_t e = t == E3_F32 ? 4 : 2;
  DenseBwdWs w{};
  if (!given && !forms_dz(t, M, K, N, true)) {  // from z in full or packed
    w.db_blocks = std::max<int64_t>(1, std::min<int64_t>(512, (M + 63) / 64));
    w.db_rows = (M + w.db_blocks - 1) / w.db_blocks;
    w.dz = up256(M * N * e);
    w.db = up256(w.db_blocks * N * 4);
  }
  // the partial sums of both products, side by side: one launch may make both
  const size_t dx = cut_bytes(dense_cut(t, M, K, N, kDx), M, K), dw = cut_bytes(dense_cut(t, K, N, M, kDw), K, N, N);
  w.part = dx + dw;
  // behind them, a W shorter than a piece
  w.total = M == 0 ? 0 : w.dz + w.db + w.part + (K * N * e < 16 ? 256 : 0);
  return w;
}

template <class T>
e3_status dense_join(const DenseArgs& a, hipStream_t st) {
  TimedLaunch t_("dense_join", st);
  const int64_t per = (a.cols + kGroup - 1) / kGroup * (kGroup / Elem<T>::V);
  hipLaunchKernelGGL(k_dense_join<T>, grid_of(((a.rows + (a.sums ? 1 : 0)) * per + 255) / 256), dim3(256), 0, st, a,
                     a.splits);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
template <class J>
e3_status dense_launch(const DenseArgs& a, const Cut& c, const Names& names, hipStream_t st) {
  TimedLaunch t_(names.tile(c.tile), st);
  const dim3 grid = grid_of(c.tiles * c.splits);
  // (packed gradient operands never get there: forms_dz; dW takes such tiles past
  // 128 columns of dz and 1e8 values of it)
  if constexpr (sizeof(typename J::T) == 2 && J::KA == kFull && J::KB == kFull && !J::SUM) {
    // Short reductions are faster by the tiles whose workgroups run two to a CU or whose
    // steps are shorter.  Direct and those, us: forward 16,384 x K x 8,192 K = 512 232 and
    // 208, 1,024 349 and 332, 1,536 435 and 451, 2,048 530 and 598, 8,192 x 4,096 x 8,192 465
    // and 561; dx of 65,536 x 512 columns from 512 59 and 49, 1,024 83 and 79, 1,536 107 and
    // 111, 2,048 132 and 152; dW 4,096 x 4,096 from 512 rows 32 and 26, 1,024 45 and 41, 2,048
    // 70 and 71, 4,096 123 and 132.
    constexpr int64_t least = 1536;
    if (c.tile == 256 && a.red >= least && a.red % 64 == 0 && direct_side(a.a, J::FA == kAlong ? 8 : a.rows) &&
        direct_side(a.b, J::FB == kAlong ? 8 : a.cols)) {
      if constexpr (J::FA == kAcross) return dense_direct_dw(a, st);
      else if constexpr (J::FB == kAlong) return dense_direct_dx(a, st);
      else return dense_direct_fwd(a, st);
    }
  }
  if constexpr (sizeof(typename J::T) == 2 && J::KA != kGradPacked && J::KB != kGradPacked) {
    if (c.tile == 256) {
      hipLaunchKernelGGL((k_dense<J, 256>), grid, dim3(TileOf<J, 256>::THREADS), 0, st, a);
      E3_HIP(hipGetLastError());
      return E3_OK;
    }
  }
  if (c.tile == 128)
    hipLaunchKernelGGL((k_dense<J, 128>), grid, dim3(TileOf<J, 128>::THREADS), 0, st, a);
  else
    hipLaunchKernelGGL((k_dense<J, 64>), grid, dim3(TileOf<J, 64>::THREADS), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
constexpr e3_dtype dtype_of(const float*) { return E3_F32; }
constexpr e3_dtype dtype_of(const __bf16*) { return E3_BF16; }
template <class J>
e3_status dense_product(DenseArgs a, float* part, const Names& names, hipStream_t st) {
  const e3_dtype t = dtype_of(static_cast<const typename J::T*>(nullptr));
  const Cut c = dense_cut(t, a.rows, a.cols, a.red, kForward);
  set_cut(a, c, part);
  const e3_status s = dense_launch<J>(a, c, names, st);
  return s != E3_OK || c.splits == 1 ? s : dense_join<typename J::T>(a, st);
}

}  // namespace
