// e3mi: dense layers, y = act(x W + b) + r, and their gradients.
//
//   z = x W + b, y = act(z) + r
//   dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum_rows dz  (dr = dy)
#include "dense_tile.h"

namespace {

struct DenseArgs {
  Side a, b;  // rows of A by columns of B over the reduction
  int64_t rows, red;
  int cols;
  int64_t chunk;  // reduction indexes per split
  int splits;
  float* part;    // partial sums [splits][rows][cols], instead of the epilogue
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

// A sum again from memory, in float32.
template <class T, Form FA, Form FB, bool QA>
__device__ __attribute__((noinline)) float dense_again(const Side& a, const Side& b, int64_t row, int col, int64_t k0,
                                                       int64_t end) {
  float sum = 0.0f;
  for (int64_t k = k0; k < end; ++k) {
    const int64_t m = FA == kAlong ? row : k, c = FA == kAlong ? k : row;
    const float u = QA ? (float)a.q[m * a.ld + c] * step8(a.c[m * a.ldc + c / kGroup])
                       : Elem<T>::one(static_cast<const T*>(a.p)[m * a.ld + c]);
    const float w = Elem<T>::one(static_cast<const T*>(b.p)[FB == kAlong ? col * b.ld + k : k * b.ld + col]);
    sum = fmaf(u, w, sum);
  }
  return sum;
}

template <class T, Form FA, Form FB, int BM, int BN, int BK, int WM, int WN, bool QA, int BUFS, int OCC>
__global__ __launch_bounds__(WM* WN* kWave, OCC) void k_dense(DenseArgs a) {
  using Tl = Tile<T, FA, FB, BM, BN, BK, WM, WN, QA, BUFS>;
  constexpr int V = Elem<T>::V;
  __shared__ __align__(16) typename Tl::Shared sh;
  const int64_t tm = (a.rows + BM - 1) / BM;
  const int tn = (a.cols + BN - 1) / BN;
  int64_t u = block_id();
  if (u >= tm * tn * a.splits) return;
  const int split = (int)(u / (tm * tn));
  u -= split * (tm * tn);
  const int64_t r0 = u / tn * BM;
  const int c0 = (int)(u % tn) * BN;
  const int64_t k0 = split * a.chunk, end = k0 + a.chunk < a.red ? k0 + a.chunk : a.red;
  Tl t;
  t.run(sh, a.a, a.b, r0, a.rows, c0, a.cols, k0, end);
  t.finish(sh, [&](int r, int lr, int c, float(&v)[V]) {
    const int64_t rowu = r0 + r, row = rowu + lr;
    const int col = c0 + c;
    const int n = row < a.rows ? a.cols - col : 0;
    if constexpr (sizeof(T) == 4) {
      float z = 0.0f;
#pragma unroll
      for (int e = 0; e < V; ++e) z += v[e] * 0.0f;
      if (z != 0.0f)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e < n && v[e] * 0.0f != 0.0f) v[e] = dense_again<T, FA, FB, QA>(a.a, a.b, row, col + e, k0, end);
    }
    if (a.part) {
      float* p = a.part + ((int64_t)split * a.rows + rowu) * a.cols + ((int64_t)lr * a.cols + col);
#pragma unroll
      for (int e = 0; e < V; e += 4) st_piece<float>(p + e, n - e, reinterpret_cast<float(&)[4]>(v[e]));
    } else {
      dense_tail<T, V>(a, rowu, lr, row < a.rows, col, v);
    }
  });
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

// The partial sums of the splits, in order, and the epilogue.
template <class T>
__global__ __launch_bounds__(256) void k_dense_join(DenseArgs a, int splits) {
  constexpr int V = Elem<T>::V;
  const int per = (a.cols + kGroup - 1) / kGroup * (kGroup / V);
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  const int col = (int)(i - row * per) * V;
  const bool ok = row < a.rows;
  float v[V] = {};
  if (ok)
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (col + e < a.cols) v[e] += a.part[((int64_t)s * a.rows + row) * a.cols + col + e];
  dense_tail<T, V>(a, row, 0, ok, col, v);
}

// dz = dy act'(z) in the type of dy (a bfloat16 dz is an operand of the matrix
// instructions, which take no more bits), and the column sums of its unrounded
// values over the block's rows.  Either output may be null.
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
// How a product is cut: tiles of bm x bn, and splits of its reduction where the
// tiles alone would leave much of the card idle.
struct Cut {
  int bm, bn, splits;
  int64_t blocks, chunk;
};
constexpr int kFill = 512;  // workgroups that fill the card
Cut dense_cut(int64_t rows, int64_t cols, int64_t red) {
  Cut c{};
  auto tiles = [&](int b, int64_t n) { return (n + b - 1) / b; };
  c.bm = c.bn = 128;
  if (tiles(128, rows) * tiles(128, cols) < kFill / 2) c.bm = c.bn = 64;
  if (cols <= 64) c.bn = 64;
  if (rows <= 64) c.bm = 64;
  if (c.bn == 64) c.bm = 64;
  if (c.bm == 64) c.bn = 64;
  const int64_t t = tiles(c.bm, rows) * tiles(c.bn, cols);
  const int64_t most = (red + 255) / 256;  // at least 256 indexes each
  int64_t s = std::max<int64_t>(1, std::min<int64_t>({kFill / std::max<int64_t>(t, 1), most, 256}));
  c.chunk = std::max<int64_t>(64, ((red + s - 1) / s + 63) / 64 * 64);
  c.splits = (int)std::max<int64_t>(1, (red + c.chunk - 1) / c.chunk);
  c.blocks = t * c.splits;
  return c;
}
size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t cut_bytes(const Cut& c, int64_t rows, int64_t cols) {
  return c.splits > 1 ? up256((size_t)c.splits * rows * cols * sizeof(float)) : 0;
}

struct DenseBwdWs {
  size_t dz, db, part, total;
  int64_t db_blocks, db_rows;
};
DenseBwdWs dense_bwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  const size_t e = t == E3_F32 ? 4 : 2;
  DenseBwdWs w{};
  w.db_blocks = std::max<int64_t>(1, std::min<int64_t>(512, (M + 63) / 64));
  w.db_rows = (M + w.db_blocks - 1) / w.db_blocks;
  w.dz = up256(M * N * e);
  w.db = up256(w.db_blocks * N * 4);
  w.part = std::max(cut_bytes(dense_cut(M, K, N), M, K), cut_bytes(dense_cut(K, N, M), K, N));
  w.total = M == 0 ? 0 : w.dz + w.db + w.part;
  return w;
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

template <class T, Form FA, Form FB, bool QA>
e3_status dense_product(DenseArgs a, float* part, const char* name, hipStream_t st) {
  const Cut c = dense_cut(a.rows, a.cols, a.red);
  a.chunk = c.chunk, a.splits = c.splits, a.part = c.splits > 1 ? part : nullptr;
  {
    TimedLaunch t_(name, st);
    constexpr bool f32 = sizeof(T) == 4;
    constexpr int BK = f32 ? 32 : 64, BUFS = f32 ? 1 : 2;
    auto* k = c.bm == 128 ? k_dense<T, FA, FB, 128, 128, BK, 2, 2, QA, BUFS, 2>
                          : k_dense<T, FA, FB, 64, 64, BK, 2, 2, QA, BUFS, 2>;
    hipLaunchKernelGGL(k, grid_of(c.blocks), dim3(256), 0, st, a);
    E3_HIP(hipGetLastError());
  }
  if (c.splits > 1) {
    TimedLaunch t_("dense_join", st);
    const int64_t per = (a.cols + kGroup - 1) / kGroup * (kGroup / Elem<T>::V);
    hipLaunchKernelGGL(k_dense_join<T>, grid_of((a.rows * per + 255) / 256), dim3(256), 0, st, a, c.splits);
    E3_HIP(hipGetLastError());
  }
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
  return dense_product<T, kAlong, kAcross, false>(a, part, "dense_fwd", st);
}

bool good_dims(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  return good_rows(t, M, K) && N >= 1 && N <= kMaxCols;
}

template <class T>
e3_status dense_bwd(RowsIn<T> x, const T* W, RowsIn<T> z, int act, const T* dy, int64_t lddy, T* dx, int64_t lddx, T* dW,
                    T* db, char* ws, int64_t M, int64_t K, int64_t N, hipStream_t st) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  const DenseBwdWs w = dense_bwd_ws(t, M, K, N);
  T* dz = reinterpret_cast<T*>(ws);
  float* dbp = reinterpret_cast<float*>(ws + w.dz);
  float* part = reinterpret_cast<float*>(ws + w.dz + w.db);
  const bool own = act != E3_ACT_NONE && (dx || dW);  // else dz is dy
  if (own || db) {
    TimedLaunch t_("dense_dz", st);
    const int per = 16 * Elem<T>::V;
    hipLaunchKernelGGL(k_dense_dz<T>, dim3((unsigned)w.db_blocks, (unsigned)((N + per - 1) / per)), dim3(256), 0, st, z,
                       act, dy, lddy, own ? dz : nullptr, db ? dbp : nullptr, M, (int)N, w.db_rows);
    E3_HIP(hipGetLastError());
  }
  if (db) {
    const e3_status s = column_sums(t, dbp, (int)w.db_blocks, 1, (int)N, db, nullptr, st);
    if (s != E3_OK) return s;
  }
  const T* d = own ? dz : dy;
  const int64_t ldd = own ? N : lddy;
  if (dx) {
    DenseArgs a{};
    a.a = {d, ldd}, a.b = {W, N}, a.rows = M, a.cols = (int)K, a.red = N;
    a.y = dx, a.ldy = lddx, a.nt = streams(t, M, K);
    const e3_status s = dense_product<T, kAlong, kAlong, false>(a, part, "dense_bwd_dx", st);
    if (s != E3_OK) return s;
  }
  if (dW) {
    DenseArgs a{};
    a.a = {x.x, x.x ? x.ld : K, x.q, x.c, (K + kGroup - 1) / kGroup}, a.b = {d, ldd};
    a.rows = K, a.cols = (int)N, a.red = M, a.y = dW, a.ldy = N;
    return x.x ? dense_product<T, kAcross, kAcross, false>(a, part, "dense_bwd_dw", st)
               : dense_product<T, kAcross, kAcross, true>(a, part, "dense_bwd_dw", st);
  }
  return E3_OK;
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
