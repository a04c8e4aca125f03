// e3mi: dense layers, y = act(x W + b) + r, and their gradients.
//
//   z = x W + b, y = act(z) + r
//   dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum_rows dz  (dr = dy)
#include "dense_tile.h"

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
template <class J, int BM, int BN>
struct TileOf {
  static constexpr bool f32 = sizeof(typename J::T) == 4;
  using type = Tile<typename J::T, J::FA, J::FB, BM, BN, f32 ? 32 : 64, 2, 2, J::KA, J::KB, J::SUM, f32 ? 1 : 2>;
};

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
  const int64_t r0 = u / tn * BM;
  const int c0 = (int)(u % tn) * BN;
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
template <class J, int BM, int BN>
__global__ __launch_bounds__(256, 2) void k_dense(DenseArgs a) {
  using Tl = typename TileOf<J, BM, BN>::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  dense_block<J, Tl, BM, BN>(a, sh, block_id());
}
// The column sums of B alone, in the order in which the product sums them.
template <class J, int BM, int BN>
__global__ __launch_bounds__(256, 2) void k_dense_sums(DenseArgs a) {
  using Tl = typename TileOf<J, BM, BN>::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  dense_block<J, Tl, BM, BN, true>(a, sh, block_id());
}
// Two products in one launch: the first `first` blocks take the first.
template <class J, class K, int BM, int BN>
__global__ __launch_bounds__(256, 2) void k_dense_two(DenseArgs a, DenseArgs b, int64_t first) {
  using Ta = typename TileOf<J, BM, BN>::type;
  using Tb = typename TileOf<K, BM, BN>::type;
  __shared__ __align__(16) union {
    typename Ta::Shared a;
    typename Tb::Shared b;
  } sh;
  const int64_t u = block_id();
  if (u < first) dense_block<J, Ta, BM, BN>(a, sh.a, u);
  else dense_block<K, Tb, BM, BN>(b, sh.b, u - first);
}

// Reductions of at most KC <= 16 (a radial basis): the weights of a thread's V
// columns stay in registers, rows go by with the next one's x in flight, and no
// LDS is used; L lanes share a row.  Bound by the write of y: 1,248,000 x 8 x 64
// float32 @THIN@ us, where the tile product took 156 (its steps are of 32).
template <class T, int L, int KC>
__global__ __launch_bounds__(256) void k_dense_thin(DenseArgs a) {
  constexpr int V = Elem<T>::V, R = 256 / L, P = KC / V > 0 ? KC / V : 1;
  const int K = (int)a.red, col = ((int)blockIdx.y * L + (int)threadIdx.x % L) * V, n = a.cols - col;
  const T* W = static_cast<const T*>(a.b.p);
  const T* x = static_cast<const T*>(a.a.p);
  float w[KC][V], bias[V] = {};
#pragma unroll
  for (int k = 0; k < KC; ++k) {
    if (k < K) {
      ld_piece<T>(W + (int64_t)k * a.cols + col, n, w[k]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) w[k][i] = 0.0f;
    }
  }
  if (a.bias) ld_piece<T>(static_cast<const T*>(a.bias) + col, n, bias);
  a.bias = nullptr;
  // U rows a thread and round, the next round's x in flight: with one, the rows'
  // latency was most of the time (@ONE@ us)
  constexpr int U = 4;
  constexpr int TR = R * U;  // rows of a round
  const int lr = threadIdx.x / L;
  typename Elem<T>::vec raw[U][P];
  auto load = [&](int64_t tile) {
    const T* xt = x + tile * TR * a.a.ld;
    const int last = a.rows - tile * TR < TR ? (int)(a.rows - tile * TR) - 1 : TR - 1;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t at = imin(lr + j * R, last) * a.a.ld;
#pragma unroll
      for (int p = 0; p < P; ++p) raw[j][p] = ld_raw<T>(xt + at + p * V, K - p * V);
    }
  };
  int64_t tile = blockIdx.x;
  if (tile * TR < a.rows) load(tile);
  for (; tile * TR < a.rows; tile += gridDim.x) {
    float v[U][V];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      float u[P][V];
#pragma unroll
      for (int p = 0; p < P; ++p) Elem<T>::get(raw[j][p], u[p]);
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = bias[i];
#pragma unroll
      for (int k = 0; k < KC; ++k)  // past K both are zero
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = fmaf(u[k / V][k % V], w[k][i], v[j][i]);
    }
    if ((tile + gridDim.x) * TR < a.rows) load(tile + gridDim.x);
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row0 = tile * TR + j * R;
      dense_tail<T, V>(a, row0, lr, row0 + lr < a.rows, col, v[j]);
    }
  }
}

// At most MR <= 8 rows: W is read once, straight to registers, and that is what
// bounds it.  A workgroup takes 32 columns; its lanes of a column piece take
// every G-th reduction index, and their sums are added over the wave and then
// over the waves in order.
template <class T, int MR>
__global__ __launch_bounds__(512) void k_dense_few(DenseArgs a) {
  constexpr int V = Elem<T>::V, C = 32 / V, G = 512 / C, WAVES = 512 / kWave;
  __shared__ float s[WAVES][MR][32];
  const int cl = threadIdx.x % C, g = threadIdx.x / C, col = (int)blockIdx.x * 32 + cl * V, n = a.cols - col;
  const int K = (int)a.red;
  const T* W = static_cast<const T*>(a.b.p);
  const T* x = static_cast<const T*>(a.a.p);
  float v[MR][V] = {};
  constexpr int U = 8;  // loads in flight
  for (int k0 = g; k0 < K; k0 += G * U) {
    typename Elem<T>::vec w[U];
    float u[U][MR];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int k = k0 + j * G;
      if (k < K) {
        w[j] = ld_raw<T>(W + (int64_t)k * a.cols + col, n);
#pragma unroll
        for (int m = 0; m < MR; ++m) u[j][m] = m < a.rows ? Elem<T>::one(x[m * a.a.ld + k]) : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (k0 + j * G < K) {
        float t[V];
        Elem<T>::get(w[j], t);
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
          for (int i = 0; i < V; ++i) v[m][i] = fmaf(u[j][m], t[i], v[m][i]);
      }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float t = sum_strided<C>(v[m][i]);
      if (threadIdx.x % kWave < C) s[threadIdx.x / kWave][m][cl * V + i] = t;
    }
  __syncthreads();
  if (threadIdx.x >= MR * C) return;
  float t[V] = {};
  for (int q = 0; q < WAVES; ++q)
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] += s[q][g][cl * V + i];
  dense_tail<T, V>(a, 0, g, g < a.rows, col, t);
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

// dz = dy act'(z) in the type of dy (a bfloat16 dz is an operand of the matrix
// instructions, which take no more bits), and the column sums of its unrounded
// values over the block's rows, for layers whose products would form dz too often
// themselves (kOnTheFly).  Either output may be null.
template <class T>
__global__ __launch_bounds__(256) void k_dense_dz(RowsIn<T> z, int act, const T* dy, int64_t lddy, T* dz, float* part,
                                                  int64_t rows, int cols, int64_t per) {
  constexpr int V = Elem<T>::V, CL = 16, RL = 256 / CL;
  __shared__ float s[RL][CL * V];
  const int cl = threadIdx.x % CL, rl = threadIdx.x / CL;
  const int col = ((int)blockIdx.y * CL + cl) * V, n = cols - col;
  const int64_t row0 = blockIdx.x * per, row1 = row0 + per < rows ? row0 + per : rows;
  float sum[V] = {};
  for (int64_t row = row0 + rl; row < row1; row += RL) {
    float u[V];
    ld_piece<T>(dy + row * lddy + col, n, u);
    if (act != E3_ACT_NONE) {
      float w[V];
      z.load(row, col, cols, w);
      act_grad_piece(act, w, u);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] += u[i];
    if (dz) st_piece<T>(dz + row * cols + col, n, u);
  }
  if (!part) return;
#pragma unroll
  for (int i = 0; i < V; ++i) s[rl][cl * V + i] = sum[i];
  __syncthreads();
  for (int i = threadIdx.x; i < CL * V; i += 256) {
    const int c = (int)blockIdx.y * CL * V + i;
    if (c >= cols) continue;
    float v = 0.0f;
#pragma unroll
    for (int r = 0; r < RL; ++r) v += s[r][i];
    part[(int64_t)blockIdx.x * cols + c] = v;
  }
}

// ------------------------------------------------------------ host
// How a product is cut: square tiles, and splits of its reduction where the
// tiles alone would leave much of the card idle.
struct Cut {
  int tile, splits;
  int64_t tiles, chunk;
};
constexpr int kFill = 512;  // workgroups that fill the card
Cut dense_cut(int64_t rows, int64_t cols, int64_t red) {
  Cut c{};
  auto tiles = [&](int b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
  c.tile = rows <= 64 || cols <= 64 || tiles(128) < kFill / 2 ? 64 : 128;
  c.tiles = tiles(c.tile);
  // at least 256 indexes a split; few tiles of few indexes take down to 64
  const int64_t least = c.tiles * (red / 256) < kFill / 8 ? 64 : 256;
  const int64_t s = std::max<int64_t>(
      1, std::min<int64_t>({kFill / std::max<int64_t>(c.tiles, 1), (red + least - 1) / least, 256}));
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
  const size_t dx = cut_bytes(dense_cut(M, K, N), M, K), dw = cut_bytes(dense_cut(K, N, M), K, N, N);
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
  auto* k = c.tile == 128 ? k_dense<J, 128, 128> : k_dense<J, 64, 64>;
  hipLaunchKernelGGL(k, grid_of(c.tiles * c.splits), dim3(256), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
template <class J>
e3_status dense_product(DenseArgs a, float* part, const char* name, hipStream_t st) {
  const Cut c = dense_cut(a.rows, a.cols, a.red);
  set_cut(a, c, part);
  const e3_status s = dense_launch<J>(a, c, name, st);
  return s != E3_OK || c.splits == 1 ? s : dense_join<typename J::T>(a, st);
}

constexpr int kThin = 16, kFew = 8;

template <class T, int L, int KC>
e3_status dense_thin(const DenseArgs& a, hipStream_t st) {
  constexpr int R = 256 / L * 4, V = Elem<T>::V;
  const int64_t tiles = (a.rows + R - 1) / R, cols = (a.cols + L * V - 1) / (L * V);
  const int64_t blocks = std::min<int64_t>(tiles, std::max<int64_t>(1, 1536 / cols));
  TimedLaunch t_("dense_thin", st);
  hipLaunchKernelGGL((k_dense_thin<T, L, KC>), dim3((unsigned)blocks, (unsigned)cols), dim3(256), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
template <class T>
e3_status dense_few(const DenseArgs& a, hipStream_t st) {
  TimedLaunch t_("dense_few", st);
  auto* k = a.rows == 1 ? k_dense_few<T, 1> : a.rows == 2 ? k_dense_few<T, 2> : a.rows <= 4 ? k_dense_few<T, 4>
                                                                                        : k_dense_few<T, kFew>;
  hipLaunchKernelGGL(k, dim3((unsigned)((a.cols + 31) / 32)), dim3(512), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

size_t dense_fwd_ws(int64_t M, int64_t K, int64_t N) {
  return M <= kFew || K <= kThin ? 0 : cut_bytes(dense_cut(M, N, K), M, N);
}
template <class T>
e3_status dense_fwd(const DenseArgs& a, float* part, hipStream_t st) {
  if (a.rows <= kFew) return dense_few<T>(a, st);
  if (a.red <= kThin) {
    constexpr int V = Elem<T>::V;
    const int pieces = (a.cols + V - 1) / V;
    auto with = [&](auto KC) {
      constexpr int kc = decltype(KC)::value;
      const int last = pieces % 64;  // lanes of a row's last column tile
      return pieces <= 8    ? dense_thin<T, 8, kc>(a, st)
             : pieces <= 16 ? dense_thin<T, 16, kc>(a, st)
             : pieces <= 32 || (last && last <= 32) ? dense_thin<T, 32, kc>(a, st)
                                                    : dense_thin<T, 64, kc>(a, st);
    };
    return a.red <= 8 ? with(std::integral_constant<int, 8>{}) : with(std::integral_constant<int, kThin>{});
  }
  return dense_product<Job<T, kAlong, kAcross, kFull, kFull, false>>(a, part, "dense_fwd", st);
}

bool good_dims(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  return good_rows(t, M, K) && N >= 1 && N <= kMaxCols;
}

// dx and dW (FLY: and db) of a layer whose operand dz is of kind KD and x of KX.
template <class T, Kind KD, Kind KX, bool FLY>
e3_status dense_bwd_products(DenseArgs x, DenseArgs w, float* part, hipStream_t st) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  using JX = Job<T, kAlong, kAlong, KD, kFull, false>;
  using JW = Job<T, kAcross, kAcross, KX, KD, FLY>;
  const bool dx = x.y, dw = w.y, db = w.sums;
  const Cut cx = dense_cut(x.rows, x.cols, x.red), cw = dense_cut(w.rows, w.cols, w.red);
  set_cut(x, cx, part);
  set_cut(w, cw, part + cut_bytes(cx, x.rows, x.cols) / sizeof(float), w.cols);
  e3_status s = E3_OK;
  if (dx && dw && cx.tile == 64 && cw.tile == 64) {
    TimedLaunch t_("dense_bwd_both", st);
    const int64_t first = cx.tiles * cx.splits;
    hipLaunchKernelGGL((k_dense_two<JX, JW, 64, 64>), grid_of(first + cw.tiles * cw.splits), dim3(256), 0, st, x, w,
                       first);
    E3_HIP(hipGetLastError());
  } else {
    if (dx) s = dense_launch<JX>(x, cx, "dense_bwd_dx", st);
    if (s == E3_OK && dw) s = dense_launch<JW>(w, cw, "dense_bwd_dw", st);
  }
  if constexpr (FLY && KX == kFull) {
    if (s == E3_OK && db && !dw) {
      TimedLaunch t_("dense_bwd_db", st);
      auto* k = cw.tile == 128 ? k_dense_sums<JW, 128, 128> : k_dense_sums<JW, 64, 64>;
      hipLaunchKernelGGL(k, grid_of((w.cols + cw.tile - 1) / cw.tile * (int64_t)cw.splits), dim3(256), 0, st, w);
      E3_HIP(hipGetLastError());
    }
  }
  if (s == E3_OK && dx && cx.splits > 1) s = dense_join<T>(x, st);
  // many partial sums of few columns take threads of their own (252 of 128 x 256: 6 us against 34)
  if (s == E3_OK && (dw || db) && cw.splits > 1 && cw.splits <= 16) s = dense_join<T>(w, st);
  if (s == E3_OK && (dw || db) && cw.splits > 16)
    s = column_sums(t, w.part, cw.splits, w.pitch, w.rows * w.cols, w.pitch, w.y, w.sums, st);
  return s;
}

template <class T>
e3_status dense_bwd(RowsIn<T> x, const T* W, RowsIn<T> z, int act, const T* dy, int64_t lddy, T* dx, int64_t lddx, T* dW,
                    T* db, char* ws, int64_t M, int64_t K, int64_t N, hipStream_t st) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  const DenseBwdWs w = dense_bwd_ws(t, M, K, N);
  const bool fly = K <= kOnTheFly;
  T* dz = reinterpret_cast<T*>(ws);
  float* dbp = reinterpret_cast<float*>(ws + w.dz);
  float* part = reinterpret_cast<float*>(ws + w.dz + w.db);
  const bool own = !fly && act != E3_ACT_NONE && (dx || dW);  // else dz is dy, or formed by the products
  if (own || (db && !fly)) {
    TimedLaunch t_("dense_dz", st);
    const int per = 16 * Elem<T>::V;
    hipLaunchKernelGGL(k_dense_dz<T>, dim3((unsigned)w.db_blocks, (unsigned)((N + per - 1) / per)), dim3(256), 0, st, z,
                       act, dy, lddy, own ? dz : nullptr, db ? dbp : nullptr, M, (int)N, w.db_rows);
    E3_HIP(hipGetLastError());
  }
  if (db && !fly) {
    const e3_status s = column_sums(t, dbp, (int)w.db_blocks, N, N, N, db, nullptr, st);
    if (s != E3_OK) return s;
  }
  DenseArgs ax{}, aw{};
  const Side d{own ? dz : dy, own ? N : lddy}, pre{z.x, z.x ? z.ld : N, z.q, z.c, (N + kGroup - 1) / kGroup};
  ax.a = d, ax.b = {W, N}, ax.pre = pre, ax.grad_act = act, ax.rows = M, ax.cols = (int)K, ax.red = N;
  ax.y = dx, ax.ldy = lddx, ax.nt = streams(t, M, K);
  aw.a = {x.x, x.x ? x.ld : K, x.q, x.c, (K + kGroup - 1) / kGroup}, aw.b = d, aw.pre = pre, aw.grad_act = act;
  aw.rows = K, aw.cols = (int)N, aw.red = M, aw.y = dW, aw.ldy = N, aw.sums = fly ? db : nullptr;
  auto run = [&](auto KD, auto FLY) {
    constexpr Kind kd = decltype(KD)::value;
    constexpr bool f = decltype(FLY)::value;
    return dW && !x.x ? dense_bwd_products<T, kd, kPacked, f>(ax, aw, part, st)
                      : dense_bwd_products<T, kd, kFull, f>(ax, aw, part, st);
  };
  using Full = std::integral_constant<Kind, kFull>;
  if (!fly) return run(Full{}, std::false_type{});
  if (act == E3_ACT_NONE) return run(Full{}, std::true_type{});
  return z.x ? run(std::integral_constant<Kind, kGradFull>{}, std::true_type{})
             : run(std::integral_constant<Kind, kGradPacked>{}, std::true_type{});
}

template <class T>
__global__ __launch_bounds__(256) void k_zero(T* p, int64_t n) {
  const int64_t i = block_id() * 256 + threadIdx.x;
  if (i < n) p[i] = (T)0.0f;
}
e3_status zeros(e3_dtype t, void* p, int64_t n, hipStream_t st) {
  if (!p) return E3_OK;
  TimedLaunch t_("dense_zero", st);
  if (t == E3_F32)
    hipLaunchKernelGGL(k_zero<float>, grid_of((n + 255) / 256), dim3(256), 0, st, static_cast<float*>(p), n);
  else
    hipLaunchKernelGGL(k_zero<__bf16>, grid_of((n + 255) / 256), dim3(256), 0, st, static_cast<__bf16*>(p), n);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

}  // namespace

extern "C" {

e3_status e3_dense_workspace_size(e3_dtype dtype, int64_t M, int64_t K, int64_t N, size_t* fwd_bytes,
                                  size_t* bwd_bytes) {
  if (!good_dims(dtype, M, K, N) || !fwd_bytes || !bwd_bytes) return E3_ERR_INVALID_ARG;
  *fwd_bytes = dense_fwd_ws(M, K, N);
  *bwd_bytes = dense_bwd_ws(dtype, M, K, N).total;
  return E3_OK;
}

e3_status e3_dense_fwd(e3_dtype dtype, const void* x, int64_t ldx, const void* W, const void* bias, const void* res,
                       int64_t ldr, e3_act act, void* y, int64_t ldy, void* z, int64_t ldz, int8_t* zq, uint8_t* zc,
                       int8_t* yq, uint8_t* yc, void* ws, size_t ws_bytes, int64_t M, int64_t K, int64_t N,
                       e3_stream stream) {
  if (!good_dims(dtype, M, K, N) || act < E3_ACT_NONE || act > E3_ACT_GELU || ldx < K || ldy < N || (res && ldr < N) ||
      (z && ldz < N) || !zq != !zc || !yq != !yc)
    return E3_ERR_INVALID_ARG;
  if (M == 0) return E3_OK;
  if (!good_ptr(dtype, x) || !good_ptr(dtype, W) || !good_ptr(dtype, y) || misaligned(dtype, bias) ||
      misaligned(dtype, res) || misaligned(dtype, z))
    return E3_ERR_INVALID_ARG;
  const size_t need = dense_fwd_ws(M, K, N);
  if (ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (need && (!ws || misaligned(E3_F32, ws))) return E3_ERR_INVALID_ARG;
  DenseArgs a{};
  a.a = {x, ldx}, a.b = {W, N}, a.rows = M, a.cols = (int)N, a.red = K;
  a.bias = bias, a.res = res, a.ldr = ldr, a.act = act, a.y = y, a.ldy = ldy, a.z = z, a.ldz = ldz, a.zq = zq;
  a.zc = zc, a.yq = yq, a.yc = yc, a.nt = streams(dtype, M, N);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  float* part = static_cast<float*>(ws);
  return dtype == E3_F32 ? dense_fwd<float>(a, part, st) : dense_fwd<__bf16>(a, part, st);
}

e3_status e3_dense_bwd(e3_dtype dtype, const void* x, int64_t ldx, const int8_t* xq, const uint8_t* xc, const void* W,
                       const void* z, int64_t ldz, const int8_t* zq, const uint8_t* zc, e3_act act, const void* dy,
                       int64_t lddy, void* dx, int64_t lddx, void* dW, void* db, void* ws, size_t ws_bytes, int64_t M,
                       int64_t K, int64_t N, e3_stream stream) {
  if (!good_dims(dtype, M, K, N) || act < E3_ACT_NONE || act > E3_ACT_GELU || (x && ldx < K) || (z && ldz < N) ||
      lddy < N || (dx && lddx < K) || !xq != !xc || !zq != !zc)
    return E3_ERR_INVALID_ARG;
  if (misaligned(dtype, x) || misaligned(dtype, W) || misaligned(dtype, z) || misaligned(dtype, dx) ||
      misaligned(dtype, dW) || misaligned(dtype, db))
    return E3_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (M == 0) {
    const e3_status s = zeros(dtype, dW, K * N, st);
    return s != E3_OK ? s : zeros(dtype, db, N, st);
  }
  if (!good_ptr(dtype, dy) || (dx && !W) || (dW && !x == !xq) || (x && xq) || (z && zq) ||
      (act != E3_ACT_NONE && !z && !zq))
    return E3_ERR_INVALID_ARG;
  const size_t need = dense_bwd_ws(dtype, M, K, N).total;
  if (ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) & 15u)) return E3_ERR_INVALID_ARG;
  auto run = [&](auto* p) {
    using T = std::remove_pointer_t<decltype(p)>;
    return dense_bwd<T>({static_cast<const T*>(x), ldx, xq, xc}, static_cast<const T*>(W),
                        {static_cast<const T*>(z), ldz, zq, zc}, act, static_cast<const T*>(dy), lddy,
                        static_cast<T*>(dx), lddx, static_cast<T*>(dW), static_cast<T*>(db), static_cast<char*>(ws), M,
                        K, N, st);
  };
  return dtype == E3_F32 ? run(static_cast<float*>(nullptr)) : run(static_cast<__bf16*>(nullptr));
}

}  // extern "C"
