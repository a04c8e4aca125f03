// Dense layers, shared by their units: arguments, the epilogue, the tile kernel
// and how a product is cut.
#pragma once
#include "dense_tile.h"

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
};
e3_status dense_bwd_f32(const DenseBwdCall& c);
e3_status dense_bwd_bf16(const DenseBwdCall& c);

namespace {

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

// What follows the sums of one piece of a row, row0 + lr with row0 uniform (so
// that a thread multiplies by a row stride once, not per piece); the lanes of a
// group of 32 columns take part together, also where rows (ok) or columns end.
template <class T, int V>
__device__ __forceinline__ void dense_tail(const DenseArgs& a, int64_t row0, int lr, bool ok, int col, float (&v)[V]) {
  static_assert(V == Elem<T>::V);
  const int n = ok ? a.cols - col : 0;
  auto at = [&](int64_t ld) { return row0 * ld + (lr * ld + col); };
  auto pack = [&](int8_t* q, uint8_t* c) {
    const int64_t groups = (a.cols + kGroup - 1) / kGroup;
    pack8_piece<V>(v, col, n, q + (row0 * a.cols + (int64_t)lr * a.cols), c + (row0 * groups + lr * groups));
  };
  float u[V];
  if (a.bias) {
    ld_piece<T>(static_cast<const T*>(a.bias) + col, n, u);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += u[i];
  }
  if (a.z) st_piece<T>(static_cast<T*>(a.z) + at(a.ldz), n, v, a.nt);
  if (a.zq) pack(a.zq, a.zc);
  act_piece(a.act, v);
  if (a.res) {
    ld_piece<T>(static_cast<const T*>(a.res) + at(a.ldr), n, u);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += u[i];
  }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = Elem<T>::round(v[i]);
  st_piece<T>(static_cast<T*>(a.y) + at(a.ldy), n, v, a.nt);
  if (a.yq) pack(a.yq, a.yc);
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
// Tiles by type and size; what a library product reaches is 1,070 TFLOP/s in
// bfloat16 and 143 in float32 (16,384 x 1,024 x 4,096).
//   bfloat16, 256 x 256: 16 waves of 64 x 64, steps of 32, two buffers, one
//     workgroup per CU: 940 (forward), 1,083 (dx), 1,056 TFLOP/s (dW); 8 waves of
//     128 x 64 760, 940, 1,019.
//   bfloat16, 128 and 64: 4 waves, steps of 64, two buffers, two workgroups and
//     more: 685, 906, 867.
//   float32, 128 x 128: one buffer of the three planes; rows along the reduction
//     with 8 waves of 32 x 64 (179 TFLOP/s; 4 of 64 x 64 161, 256 x 256 145),
//     across with 4 (208; 8 193).
template <class J, int B>
struct TileOf {
  static constexpr bool f32 = sizeof(typename J::T) == 4;
  static constexpr int WM = B == 256 || (f32 && B == 128 && J::FA == kAlong) ? 4 : 2, WN = B == 256 ? 4 : 2;
  static constexpr int BK = f32 || B == 256 ? 32 : 64, THREADS = WM * WN * kWave, OCC = B == 256 ? 4 : 2;
  using type = Tile<typename J::T, J::FA, J::FB, B, B, BK, WM, WN, J::KA, J::KB, J::SUM, f32 ? 1 : 2>;
};

// Which tile block u of tm x tn takes: blocks go round robin to the XCDs, so an
// XCD takes a contiguous eighth, eight row tiles by eight column tiles running
// together, which share their operands in its L2.
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
  t.finish(sh, [&](int r, int lr, int c, float(&v)[V]) {
    const int64_t rowu = r0 + r, row = rowu + lr;
    const int col = c0 + c;
    const int n = row < a.rows ? a.cols - col : 0;
    if constexpr (sizeof(T) == 4) {
      float z = 0.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) z += v[e] * 0.0f;
      if (z != 0.0f) {
        float t[V];
#pragma clang loop unroll(disable)
        for (int e = 0; e < V; ++e) {
          const float again = e < n ? dense_again<T, J::FA, J::FB, J::KA, J::KB>(a, row, col + e, k0, end) : 0.0f;
#pragma unroll
          for (int q = 0; q < V; ++q) t[q] = q == e ? again : t[q];
        }
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = v[e] * 0.0f != 0.0f ? t[e] : v[e];
      }
    }
    if (a.part) {
      float* p = a.part + (split * a.pitch + rowu * a.cols) + ((int64_t)lr * a.cols + col);
#pragma unroll
      for (int e = 0; e < V; e += 4) st_piece<float>(p + e, n - e, reinterpret_cast<float(&)[4]>(v[e]));
    } else {
      dense_tail<T, V>(a, rowu, lr, row < a.rows, col, v);
    }
  });
}
template <class J, int B>
__global__ __launch_bounds__((TileOf<J, B>::THREADS), (TileOf<J, B>::OCC)) void k_dense(DenseArgs a) {
  using Tl = typename TileOf<J, B>::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  dense_block<J, Tl, B, B>(a, sh, block_id());
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
  int tile, splits;
  int64_t tiles, chunk;
};
constexpr int kFill = 512;  // workgroups of the smaller tiles that fill the card
Cut dense_cut(e3_dtype t, int64_t rows, int64_t cols, int64_t red) {
  Cut c{};
  auto tiles = [&](int b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
  c.tile = rows <= 64 || cols <= 64 || tiles(128) < kFill / 2 ? 64 : 128;
  int64_t fill = kFill;
  if (t == E3_BF16 && rows > 128 && cols > 128) {
    // rounds of the card by the time of one: four times the work of a 128 x 128
    // tile, of which two run on a CU at 0.78 of the rate
    auto time = [&](int64_t n, int64_t slots, double round) {
      const int64_t s = std::max<int64_t>(1, std::min(slots / n, red / 512));
      return (double)((n * s + slots - 1) / slots) * round / (double)s;
    };
    if (time(tiles(256), 256, 4.0) <= time(tiles(128), 512, 2.56)) c.tile = 256, fill = 256;
  }
  c.tiles = tiles(c.tile);
  // at least 256 indexes a split; few tiles of few indexes take down to 64
  const int64_t least = c.tiles * (red / 256) < kFill / 8 ? 64 : c.tile == 256 ? 512 : 256;
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

// The products of the backward form dz from dy and z on the way to LDS: once per
// 128 columns of x, so up to this many; wider layers write dz once.  (Two rounds
// of an activation's derivative cost less than dz's way to memory and back.)
constexpr int64_t kOnTheFly = 256;

struct DenseBwdWs {
  size_t dz, db, part, total;
  int64_t db_blocks, db_rows;
};
DenseBwdWs dense_bwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  const size_t e = t == E3_F32 ? 4 : 2;
  DenseBwdWs w{};
  if (K > kOnTheFly) {
    w.db_blocks = std::max<int64_t>(1, std::min<int64_t>(512, (M + 63) / 64));
    w.db_rows = (M + w.db_blocks - 1) / w.db_blocks;
    w.dz = up256(M * N * e);
    w.db = up256(w.db_blocks * N * 4);
  }
  // dx's own partial sums are joined before dW's are made, unless one launch makes both
  const size_t dx = cut_bytes(dense_cut(t, M, K, N), M, K), dw = cut_bytes(dense_cut(t, K, N, M), K, N, N);
  w.part = dx + dw;
  w.total = M == 0 ? 0 : w.dz + w.db + w.part;
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
e3_status dense_launch(const DenseArgs& a, const Cut& c, const char* name, hipStream_t st) {
  TimedLaunch t_(name, st);
  const dim3 grid = grid_of(c.tiles * c.splits);
  if constexpr (sizeof(typename J::T) == 2) {
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
e3_status dense_product(DenseArgs a, float* part, const char* name, hipStream_t st) {
  const Cut c = dense_cut(dtype_of(static_cast<const typename J::T*>(nullptr)), a.rows, a.cols, a.red);
  set_cut(a, c, part);
  const e3_status s = dense_launch<J>(a, c, name, st);
  return s != E3_OK || c.splits == 1 ? s : dense_join<typename J::T>(a, st);
}

}  // namespace
