// e3mi: dense layers, y = act(x W + b) + r, and their gradients.
//
//   z = x W + b, y = act(z) + r
//   dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum_rows dz  (dr = dy)
#include "layers.h"

namespace {

constexpr int kTile = 64, kStep = 16;

struct DenseArgs {
  // operands of the product: rows of A by columns of B over a reduction axis
  const void *a, *b;
  int64_t a_row, a_red, b_red, b_col;  // element strides
  const int8_t* aq;                    // A packed (its rows run along the reduction: dW's x)
  const uint8_t* ac;
  int64_t rows, red;
  int cols;
  int packed_cols;
  int64_t chunk;  // reduction indexes per split (blockIdx.z)
  float* part;    // partial sums [splits][rows][cols], instead of the epilogue
  // epilogue
  const void *bias, *res;
  void *y, *z;
  int8_t *zq, *yq;
  uint8_t *zc, *yc;
  int64_t ldr, ldy, ldz;
  int act;
};

// What follows the sums of one piece of a row; the lanes of a group of 32
// columns take part together, also where the row (row_ok) or columns end.
template <class T, int V>
__device__ __forceinline__ void dense_tail(const DenseArgs& a, int64_t row, bool row_ok, int col, float (&v)[V]) {
  static_assert(V == Elem<T>::V);
  const int n = row_ok ? a.cols - col : 0;
  const int64_t groups = (a.cols + kGroup - 1) / kGroup;
  float u[V];
  if (a.bias) {
    ld_piece<T>(static_cast<const T*>(a.bias) + col, n, u);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += u[i];
  }
  if (a.z) st_piece<T>(static_cast<T*>(a.z) + row * a.ldz + col, n, v);
  if (a.zq) pack8_piece<V>(v, col, n, a.zq + row * a.cols, a.zc + row * groups);
  if (a.act != E3_ACT_NONE)
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_of(a.act, v[i]);
  if (a.res) {
    ld_piece<T>(static_cast<const T*>(a.res) + row * a.ldr + col, n, u);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += u[i];
  }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = Elem<T>::round(v[i]);
  st_piece<T>(static_cast<T*>(a.y) + row * a.ldy + col, n, v);
  if (a.yq) pack8_piece<V>(v, col, n, a.yq + row * a.cols, a.yc + row * groups);
}

template <class T>
__global__ __launch_bounds__(256) void k_dense(DenseArgs a) {
  __shared__ float sA[kStep][kTile + 4], sB[kStep][kTile + 4], sC[kTile][kTile + 4];
  const int tid = threadIdx.x, tr = tid / 16 * 4, tc = tid % 16 * 4;
  const int64_t row0 = (int64_t)blockIdx.x * kTile;
  const int col0 = (int)blockIdx.y * kTile;
  const int64_t r0 = blockIdx.z * a.chunk, r1 = r0 + a.chunk < a.red ? r0 + a.chunk : a.red;
  const T* A = static_cast<const T*>(a.a);
  const T* B = static_cast<const T*>(a.b);
  float acc[4][4] = {};
  for (int64_t r = r0; r < r1; r += kStep) {
    for (int i = tid; i < kStep * kTile; i += 256) {
      const int k = i % kStep, m = i / kStep, k2 = i / kTile, n = i % kTile;
      float u = 0.0f, w = 0.0f;
      if (row0 + m < a.rows && r + k < r1) {
        if (a.aq) {
          const int64_t at = r + k;
          const int col = (int)(row0 + m);
          u = (float)a.aq[at * a.packed_cols + col] *
              step8(a.ac[at * ((a.packed_cols + kGroup - 1) / kGroup) + col / kGroup]);
        } else {
          u = Elem<T>::one(A[(row0 + m) * a.a_row + (r + k) * a.a_red]);
        }
      }
      if (col0 + n < a.cols && r + k2 < r1) w = Elem<T>::one(B[(r + k2) * a.b_red + (col0 + n) * a.b_col]);
      sA[k][m] = u;
      sB[k2][n] = w;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sA[k][tr + i], sB[k][tc + j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sC[tr + i][tc + j] = acc[i][j];
  __syncthreads();
  constexpr int V = Elem<T>::V, P = kTile / V;
  for (int i = tid; i < kTile * P; i += 256) {
    const int m = i / P, c = i % P * V;
    const int64_t row = row0 + m;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = sC[m][c + e];
    if (a.part) {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (row < a.rows && col0 + c + e < a.cols)
          a.part[((int64_t)blockIdx.z * a.rows + row) * a.cols + col0 + c + e] = v[e];
    } else {
      dense_tail<T, V>(a, row, row < a.rows, col0 + c, v);
    }
  }
}

// The partial sums of the splits, in order, and the epilogue.
template <class T>
__global__ __launch_bounds__(256) void k_dense_join(DenseArgs a, int splits) {
  constexpr int V = Elem<T>::V;
  const int per = (a.cols + kGroup - 1) / kGroup * (kGroup / V);
  const int64_t i = block_id() * 256 + threadIdx.x, row = i / per;
  const int col = (int)(i - row * per) * V;
  const bool ok = row < a.rows;
  float v[V] = {};
  if (ok)
    for (int s = 0; s < splits; ++s)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (col + e < a.cols) v[e] += a.part[((int64_t)s * a.rows + row) * a.cols + col + e];
  dense_tail<T, V>(a, row, ok, col, v);
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
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] *= act_grad(act, w[i]);
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
int64_t tiles(int64_t n) { return (n + kTile - 1) / kTile; }
// Splits of a reduction of `red` over a grid of `blocks` tiles: enough to fill
// the card, each of at least 64 indexes.
int64_t dense_splits(int64_t blocks, int64_t red) {
  return std::max<int64_t>(1, std::min<int64_t>({1024 / std::max<int64_t>(blocks, 1), (red + 63) / 64, 64}));
}
int64_t dense_chunk(int64_t red, int64_t splits) { return ((red + splits - 1) / splits + 63) / 64 * 64; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct DenseBwdWs {
  size_t dz, db, dw, total;
  int64_t db_blocks, db_rows, dw_splits;
};
DenseBwdWs dense_bwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  const size_t e = t == E3_F32 ? 4 : 2;
  DenseBwdWs w{};
  w.db_blocks = std::max<int64_t>(1, std::min<int64_t>(512, (M + 63) / 64));
  w.db_rows = (M + w.db_blocks - 1) / w.db_blocks;
  w.dw_splits = dense_splits(tiles(K) * tiles(N), M);
  w.dz = up256(M * N * e);
  w.db = up256(w.db_blocks * N * 4);
  w.dw = w.dw_splits > 1 ? up256(w.dw_splits * K * N * 4) : 0;
  w.total = M == 0 ? 0 : w.dz + w.db + w.dw;
  return w;
}

template <class T>
e3_status dense_product(DenseArgs a, int64_t splits, float* part, const char* name, hipStream_t st) {
  a.chunk = dense_chunk(a.red, splits);
  splits = (a.red + a.chunk - 1) / a.chunk;
  a.part = splits > 1 ? part : nullptr;
  {
    TimedLaunch t_(name, st);
    hipLaunchKernelGGL(k_dense<T>, dim3((unsigned)tiles(a.rows), (unsigned)tiles(a.cols), (unsigned)splits), dim3(256),
                       0, st, a);
    E3_HIP(hipGetLastError());
  }
  if (splits > 1) {
    TimedLaunch t_("dense_join", st);
    const int64_t per = (a.cols + kGroup - 1) / kGroup * (kGroup / Elem<T>::V);
    hipLaunchKernelGGL(k_dense_join<T>, grid_of((a.rows * per + 255) / 256), dim3(256), 0, st, a, (int)splits);
    E3_HIP(hipGetLastError());
  }
  return E3_OK;
}

size_t dense_fwd_ws(int64_t M, int64_t K, int64_t N) {
  const int64_t s = dense_splits(tiles(M) * tiles(N), K);
  return M == 0 || s == 1 ? 0 : up256(s * M * N * 4);
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
  float* dwp = reinterpret_cast<float*>(ws + w.dz + w.db);
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
    a.a = d, a.a_row = ldd, a.a_red = 1, a.b = W, a.b_red = 1, a.b_col = N, a.rows = M, a.cols = (int)K, a.red = N;
    a.y = dx, a.ldy = lddx;
    const e3_status s = dense_product<T>(a, 1, nullptr, "dense_bwd_dx", st);
    if (s != E3_OK) return s;
  }
  if (dW) {
    DenseArgs a{};
    a.a = x.x, a.a_row = 1, a.a_red = x.ld, a.aq = x.x ? nullptr : x.q, a.ac = x.c, a.packed_cols = (int)K;
    a.b = d, a.b_red = ldd, a.b_col = 1, a.rows = K, a.cols = (int)N, a.red = M, a.y = dW, a.ldy = N;
    return dense_product<T>(a, w.dw_splits, dwp, "dense_bwd_dw", st);
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
  a.a = x, a.a_row = ldx, a.a_red = 1, a.b = W, a.b_red = N, a.b_col = 1, a.rows = M, a.cols = (int)N, a.red = K;
  a.bias = bias, a.res = res, a.ldr = ldr, a.act = act, a.y = y, a.ldy = ldy, a.z = z, a.ldz = ldz, a.zq = zq;
  a.zc = zc, a.yq = yq, a.yc = yc;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int64_t splits = dense_splits(tiles(M) * tiles(N), K);
  float* part = static_cast<float*>(ws);
  return dtype == E3_F32 ? dense_product<float>(a, splits, part, "dense_fwd", st)
                         : dense_product<__bf16>(a, splits, part, "dense_fwd", st);
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
