// e3mi: dense layers, y = act(x W + b) + r, and their gradients.
//
//   z = x W + b, y = act(z) + r
//   dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum_rows dz  (dr = dy)
//
// This unit holds the forward and the C entry points; the tile product is in
// dense_tile.h, the backward in dense_bwd.h (a unit per type).
#include "dense.h"

namespace {

// Reductions of at most KC <= 16 (a radial basis): the weights of a thread's V
// columns stay in registers, rows go by with the next one's x in flight, and no
// LDS is used; L lanes share a row.  Bound by the write of y: 1,248,000 x 8 x 64
// float32 with silu 60 us (6.0 TB/s; 320 MB of zeros take 47), where the tile
// product took 156 (its steps are of 32).
template <class T, int L, int KC, bool FAST>
__global__ __launch_bounds__(256) void k_dense_thin(DenseArgs a) {
  constexpr int V = Elem<T>::V, R = 256 / L, P = KC / V > 0 ? KC / V : 1;
  const int K = (int)a.red, col = ((int)blockIdx.y * L + (int)threadIdx.x % L) * V, n = a.cols - col;
  const T* W = static_cast<const T*>(a.b.p);
  const T* x = static_cast<const T*>(a.a.p);
  float w[KC][V];
  const Tail<T> tail(a, col);
#pragma unroll
  for (int k = 0; k < KC; ++k) {
    if (k < K) {
      ld_piece<T>(W + (int64_t)k * a.cols + col, n, w[k]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) w[k][i] = 0.0f;
    }
  }
  // U rows a thread and round, the next round's x in flight (one row a round: 129
  // us against 117 before the stores were non-temporal)
  constexpr int U = 4;
  constexpr int TR = R * U;  // rows of a round
  const int lr = threadIdx.x / L;
  typename Elem<T>::vec raw[U][P];
  auto load = [&](auto fast, int64_t tile) {
    constexpr bool F = decltype(fast)::value;
    const T* xt = x + tile * TR * a.a.ld;
    const int last = F ? TR - 1 : a.rows - tile * TR < TR ? (int)(a.rows - tile * TR) - 1 : TR - 1;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t at = imin(lr + j * R, last) * a.a.ld;
#pragma unroll
      for (int p = 0; p < P; ++p) raw[j][p] = ld_raw<T>(xt + at + p * V, F ? V : K - p * V);
    }
  };
  float v[U][V];
  auto sums = [&]() {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      float u[P][V];
#pragma unroll
      for (int p = 0; p < P; ++p) Elem<T>::get(raw[j][p], u[p]);
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = 0.0f;
#pragma unroll
      for (int k = 0; k < KC; ++k)  // past K both are zero
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = fmaf(u[k / V][k % V], w[k][i], v[j][i]);
    }
  };
  auto out = [&](auto fast, int64_t tile, const typename Tail<T>::Raw (&res)[U]) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row0 = tile * TR + j * R;
      tail.template out<decltype(fast)::value>(a, row0, lr, row0 + lr < a.rows, col, res[j], v[j]);
    }
  };
  auto residuals = [&](int64_t tile, typename Tail<T>::Raw (&res)[U]) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int64_t row0 = tile * TR + j * R;
      res[j] = Tail<T>::residual(a, row0, lr, row0 + lr < a.rows, col);
    }
  };
  // FAST: whole tiles by a loop without branches around loads and stores, and what
  // is left of the rows after it
  const int64_t tiles = FAST ? a.rows / TR : (a.rows + TR - 1) / TR;
  const std::integral_constant<bool, FAST> fast;
  const int64_t tile0 = blockIdx.x;
  typename Tail<T>::Raw res[U];
  if (tile0 < tiles) {
    // a round ends with loads and begins with stores, so that its wait for the
    // loads of the one before leaves its own stores in flight; tiles past the end
    // load the last one again
    auto at = [&](int64_t t) { return t < tiles ? t : tiles - 1; };
    load(fast, tile0);
    sums();
    load(fast, at(tile0 + gridDim.x));
    for (int64_t tile = tile0; tile < tiles; tile += gridDim.x) {
      if (!FAST) residuals(tile, res);
      out(fast, tile, res);
      sums();
      load(fast, at(tile + 2 * (int64_t)gridDim.x));
    }
  }
  if (FAST && tiles * TR < a.rows && blockIdx.x == tiles % gridDim.x) {
    load(std::false_type{}, tiles);
    residuals(tiles, res);
    sums();
    out(std::false_type{}, tiles, res);
  }
}

// At most MR <= 8 rows: W is read once, straight to registers, and that is what
// bounds it (one row of 1,024 to 4,096 in bfloat16 5.8 us, of which a launch is
// about half).  A workgroup takes 32 columns; its lanes of a column piece take
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

// ------------------------------------------------------------ host
constexpr int kThin = 16, kFew = 8;

template <class T, int L, int KC>
e3_status dense_thin(const DenseArgs& a, hipStream_t st) {
  constexpr int R = 256 / L * 4, V = Elem<T>::V;
  const int64_t tiles = (a.rows + R - 1) / R, cols = (a.cols + L * V - 1) / (L * V);
  const int64_t blocks = std::min<int64_t>(tiles, std::max<int64_t>(1, 1536 / cols));
  TimedLaunch t_("dense_thin", st);
  auto* k = Tail<T>::plain(a) && a.red == KC && a.cols % (L * V) == 0 ? k_dense_thin<T, L, KC, true> : k_dense_thin<T, L, KC, false>;
  hipLaunchKernelGGL(k, dim3((unsigned)blocks, (unsigned)cols), dim3(256), 0, st, a);
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

size_t dense_fwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  const bool p = t == E3_F32 ? panel<float>(M, N, K) : panel<__bf16>(M, N, K);
  return M <= kFew || K <= kThin || p ? 0 : cut_bytes(dense_cut(t, M, N, K, kForward), M, N);
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
  using J = Job<T, kAlong, kAcross, kFull, kFull, false>;
  if (panel<T>(a.rows, a.cols, a.red)) return dense_panel<J>(a, kNamesFwd, st);
  return dense_product<J>(a, part, kNamesFwd, st);
}

bool good_dims(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  return good_rows(t, M, K) && N >= 1 && N <= kMaxCols;
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
  *fwd_bytes = dense_fwd_ws(dtype, M, K, N);
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
  const size_t need = dense_fwd_ws(dtype, M, K, N);
  if (ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (need && (!ws || misaligned(E3_F32, ws))) return E3_ERR_INVALID_ARG;
  DenseArgs a{};
  a.a = {x, ldx, nullptr, nullptr, 0, (M - 1) * ldx + K}, a.b = {W, N, nullptr, nullptr, 0, K * N};
  a.rows = M, a.cols = (int)N, a.red = K;
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
  const DenseBwdCall c{dtype, x,  W,  z,  dy, xq,  zq,  xc,  zc,   dx,   dW, db, static_cast<char*>(ws),
                       ldx,   ldz, lddy, lddx, M, K, N, act, st};
  return dtype == E3_F32 ? dense_bwd_f32(c) : dense_bwd_bf16(c);
}

}  // extern "C"
