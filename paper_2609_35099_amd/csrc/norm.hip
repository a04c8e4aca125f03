// e3mi: layer norm (forward, backward, the weight gradients) and 8-bit
// activation checkpoints.
//
//   y = (x - mean) rstd g + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   with n = (x - mean) rstd and a = dy g:
//   dx = rstd (a - mean(a) - n mean(a n)),  dg = sum_rows dy n,  db = sum_rows dy
//
// All of it is bound by memory: a row is read once, kept in registers through
// both passes over it and written once, together with its 8-bit checkpoint where
// one is asked for.  The first pass gives the mean m as a float32, which is off by
// up to 2^-24 of itself and its sum's roundings; the second sums the deviations
// x - m (exact near m) and their squares: with c the mean of the deviations, the
// row's mean is m + c, its deviations x - m - c and its variance that of x - m
// less c^2.  Without c, a mean 3,000 times the deviation moved y by 2e-4; with it,
// float32 rows take up to 4% longer (20,000 x 1,024 29.2 us without, 30.3 with).
// bfloat16 rows go without: their values have 8 bits, so where the mean is 256
// times the deviation (m off by 1e-4 of it, y's last bit 4e-3) little else is left
// of them.  The backward takes the mean as float32, whose rounding shifts its n.
// L lanes share a row, J 16-byte pieces each; narrow rows take part of a wave, wide
// ones a workgroup, and rows past the registers are read again for each pass.
//
// One MI355X, us per call in a row of calls: 65,536 x 1,024 bfloat16 forward with
// statistics and x in 8 bits 65 (5.2 TB/s), backward from x in 8 bits 63, of which dx
// alone 50 (6.7 TB/s, x's 8 bits from the last-level cache); 100,003 x 515 float32
// forward 69 (5.9 TB/s), backward 130, dx alone 117 (5.3).  Packing 65,536 x 2,048
// bfloat16 80 (5.1), unpacking 60 (6.8).
#include "layers.h"

namespace {

constexpr int kNormThreads = 256;

struct NormArgs {
  const void *x, *gamma, *beta, *dy;
  void *y, *dx;
  float *mean, *rstd;
  const int8_t* xq_in;
  const uint8_t* xc_in;
  int8_t *xq, *yq;
  uint8_t *xc, *yc;
  float* part;  // [blocks][2][cols]: partial dg, db
  int64_t ldx, ldy, lddx, rows;
  int cols, blocks;
  float eps;
  bool nt;  // y or dx streams
};

// Sums over the L lanes of a row: part of a wave, or the whole workgroup (then
// every thread calls it; `s` holds a value per wave).
template <int L>
__device__ __forceinline__ float row_sum(float v, float* s) {
  if constexpr (L <= kWave) return sum_lanes<L>(v);
  v = sum_lanes<kWave>(v);
  if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < L / kWave; ++w) v += s[w];
  __syncthreads();
  return v;
}

// Two sums at once, to u and v (s: two values per wave).
template <int L>
__device__ __forceinline__ void row_sums(float& u, float& v, float* s) {
  if constexpr (L <= kWave) {
    u = sum_lanes<L>(u), v = sum_lanes<L>(v);
  } else {
    constexpr int W = L / kWave;
    u = sum_lanes<kWave>(u), v = sum_lanes<kWave>(v);
    if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = u, s[W + threadIdx.x / kWave] = v;
    __syncthreads();
    u = 0.0f, v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) u += s[w], v += s[W + w];
    __syncthreads();
  }
}

// J > 0: the row's pieces stay in registers.  J = 0: any width, piece by piece.
template <int L>
constexpr int kNormFwdThreads = L <= kNormThreads ? kNormThreads : L;
template <class T, int L, int J>
__global__ __launch_bounds__(kNormFwdThreads<L>) void k_norm_fwd(NormArgs a) {
  constexpr int V = Elem<T>::V, R = kNormFwdThreads<L> / L, U = J > 0 ? J : 1;
  __shared__ float s[2 * kNormFwdThreads<L> / kWave];
  const int lane = threadIdx.x % L, cols = a.cols;
  const int64_t row = block_id() * R + threadIdx.x / L;
  if (row >= a.rows) return;  // whole rows leave: no lane of another row's group
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const int pieces = J > 0 ? J : (cols + L * V - 1) / (L * V);
  float v[U][V];
  auto piece = [&](int j) -> float(&)[V] {
    if constexpr (J > 0) {
      return v[j];
    } else {
      const int col = (j * L + lane) * V;
      ld_piece<T>(x + col, cols - col, v[0]);
      return v[0];
    }
  };
  if constexpr (J > 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int col = (j * L + lane) * V;
      ld_piece<T>(x + col, cols - col, v[j]);
    }
  }
  float sum = 0.0f;
#pragma unroll U
  for (int j = 0; j < pieces; ++j) {
    float(&u)[V] = piece(j);
#pragma unroll
    for (int i = 0; i < V; ++i) sum += u[i];
  }
  const float mean = row_sum<L>(sum, s) / (float)cols;
  constexpr bool DEV = sizeof(T) == 4;
  float dev = 0.0f, sq = 0.0f;
#pragma unroll U
  for (int j = 0; j < pieces; ++j) {
    float(&u)[V] = piece(j);
    const int n = cols - (j * L + lane) * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float d = i < n ? u[i] - mean : 0.0f;
      if constexpr (DEV) dev += d;
      sq += d * d;
    }
  }
  if constexpr (DEV) row_sums<L>(dev, sq, s);
  else sq = row_sum<L>(sq, s);
  dev /= (float)cols;
  float var = sq / (float)cols;
  if constexpr (DEV) {
    var -= dev * dev;
    if (var < 0.0f) var = 0.0f;  // (a NaN stays)
  }
  const float rstd = 1.0f / sqrtf(var + a.eps);
  if (lane == 0) {
    if (a.mean) a.mean[row] = mean + dev;
    if (a.rstd) a.rstd[row] = rstd;
  }
  const T* gamma = static_cast<const T*>(a.gamma);
  const T* beta = static_cast<const T*>(a.beta);
  const int64_t groups = (cols + kGroup - 1) / kGroup;
  dev *= -rstd;
#pragma unroll U
  for (int j = 0; j < pieces; ++j) {
    float(&u)[V] = piece(j);
    const int col = (j * L + lane) * V, n = cols - col;
    if (a.xq) pack8_piece<V>(u, col, n, a.xq + row * cols, a.xc + row * groups);
    float g[V], b[V];
    if (gamma) ld_piece<T>(gamma + col, n, g);
    if (beta) ld_piece<T>(beta + col, n, b);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float w = DEV ? fmaf(u[i] - mean, rstd, dev) : (u[i] - mean) * rstd;
      const float t = gamma ? w * g[i] : w;
      u[i] = Elem<T>::round(beta ? t + b[i] : t);
    }
    st_piece<T>(static_cast<T*>(a.y) + row * a.ldy + col, n, u, a.nt);
    if (a.yq) pack8_piece<V>(u, col, n, a.yq + row * cols, a.yc + row * groups);
  }
}

// dx, and per workgroup the sums of dy n and dy over its rows (rows blockIdx.x
// R + i, then every gridDim.x R).  The next row's pieces are in flight while a
// row is worked on.  Workgroups are large and few, so that little is left for
// the sum over them: 512 threads where a row takes at most a wave (1,024 leave
// too few registers), one row where it takes more.
// Which products are fused into sums is written out: left to the compiler, it
// differs between the instances, and a gradient asked for alone (another instance
// where dx streams) had other bits than beside dx.
template <int L>
constexpr int kNormBwdThreads = L <= kWave ? 512 : L;
template <class T, int L, int J, bool Q, bool FAST>
__global__ __launch_bounds__(kNormBwdThreads<L>) void k_norm_bwd(NormArgs a) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V, NT = kNormBwdThreads<L>, R = NT / L;
  using In = RowsIn<T>;
  __shared__ float s[NT / kWave];
  __shared__ float fold[R > 1 ? NT * V : 1];
  const int lane = threadIdx.x % L, cols = a.cols;
  const In xs{static_cast<const T*>(a.x), a.ldx, a.xq_in, a.xc_in};
  const T* dyp = static_cast<const T*>(a.dy);
  const T* gamma = static_cast<const T*>(a.gamma);
  float dg[J][V] = {}, db[J][V] = {};
  const int64_t stride = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
  typename In::template Raw<Q> xr[J];
  typename Elem<T>::vec dr[J], gr[J];
  if (gamma)
#pragma unroll
    for (int j = 0; j < J; ++j) gr[j] = ld_raw<T>(gamma + (j * L + lane) * V, cols - (j * L + lane) * V);
  float mean = 0.0f, rstd = 0.0f, x[J][V], dy[J][V];
  // FAST: every piece is whole and dx streams.  A round then has no branch around
  // its stores, and as it ends with loads, its wait for those of the round before
  // leaves its own stores in flight.
  auto load = [&](int64_t r) {
    if (r >= a.rows) r = a.rows - 1;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int col = (j * L + lane) * V;
      xr[j] = xs.template raw<Q>(r, col, FAST ? L * J * V : cols);
      dr[j] = ld_raw<T>(dyp + r * a.ldy + col, FAST ? V : cols - col);
    }
    mean = a.mean[r], rstd = a.rstd[r];
  };
  auto take = [&](float& m, float& rs) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      In::template get<Q>(xr[j], x[j]);
      Elem<T>::get(dr[j], dy[j]);
    }
    m = mean, rs = rstd;
  };
  float m = 0.0f, rs = 0.0f;
  if (row < a.rows) {
    load(row);
    take(m, rs);
    load(row + stride);
  }
  for (; row < a.rows; row += stride) {
    float c0 = 0.0f, c1 = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int col = (j * L + lane) * V, n = FAST ? V : cols - col;
      float g[V];
      if (gamma) Elem<T>::get(gr[j], g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        // columns past the end have dy = 0: x there must not turn them into NaN
        x[j][i] = i < n ? (x[j][i] - m) * rs : 0.0f;
        dg[j][i] = fmaf(dy[j][i], x[j][i], dg[j][i]);
        db[j][i] += dy[j][i];
        if (gamma) dy[j][i] *= g[i];
        c0 += dy[j][i];
        c1 = fmaf(dy[j][i], x[j][i], c1);
      }
    }
    if (FAST || a.dx) {
      c0 = row_sum<L>(c0, s) / (float)cols;
      c1 = row_sum<L>(c1, s) / (float)cols;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int col = (j * L + lane) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) dy[j][i] = rs * fmaf(-x[j][i], c1, dy[j][i] - c0);
        st_piece<T>(static_cast<T*>(a.dx) + row * a.lddx + col, FAST ? V : cols - col, dy[j], FAST || a.nt);
      }
    }
    take(m, rs);
    load(row + 2 * stride);
  }
  if (!a.part) return;
  float* out = a.part + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = k ? db[j][i] : dg[j][i];
      if constexpr (R > 1) {
        // the rows of the workgroup, in order
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) fold[threadIdx.x * V + i] = v[i];
        __syncthreads();
        if (threadIdx.x >= L) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] += fold[(r * L + lane) * V + i];
      }
      const int col = (j * L + lane) * V;
      st_piece<float>(out + (int64_t)k * cols + col, cols - col, reinterpret_cast<float(&)[4]>(v[0]));
      if constexpr (V == 8)
        st_piece<float>(out + (int64_t)k * cols + col + 4, cols - col - 4, reinterpret_cast<float(&)[4]>(v[4]));
    }
  }
}

// Rows too wide for registers: dx of one row, read twice.
template <class T>
__global__ __launch_bounds__(kNormThreads) void k_norm_bwd_wide(NormArgs a) {
  constexpr int V = Elem<T>::V, L = kNormThreads;
  __shared__ float s[kNormThreads / kWave];
  const int lane = threadIdx.x, cols = a.cols;
  const int64_t row = block_id();
  if (row >= a.rows) return;
  const RowsIn<T> xs{static_cast<const T*>(a.x), a.ldx, a.xq_in, a.xc_in};
  const T* gamma = static_cast<const T*>(a.gamma);
  const T* dyr = static_cast<const T*>(a.dy) + row * a.ldy;
  const float mean = a.mean[row], rstd = a.rstd[row];
  auto load = [&](int col, float(&x)[V], float(&u)[V]) {
    const int n = cols - col;
    xs.load(row, col, cols, x);
    ld_piece<T>(dyr + col, n, u);
    if (gamma) {
      float g[V];
      ld_piece<T>(gamma + col, n, g);
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] *= g[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = i < n ? (x[i] - mean) * rstd : 0.0f;
  };
  float c0 = 0.0f, c1 = 0.0f, x[V], u[V];
  for (int col = lane * V; col < cols; col += L * V) {
    load(col, x, u);
#pragma unroll
    for (int i = 0; i < V; ++i) c0 += u[i], c1 += u[i] * x[i];
  }
  c0 = row_sum<L>(c0, s) / (float)cols;
  c1 = row_sum<L>(c1, s) / (float)cols;
  for (int col = lane * V; col < cols; col += L * V) {
    load(col, x, u);
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = rstd * (u[i] - c0 - x[i] * c1);
    st_piece<T>(static_cast<T*>(a.dx) + row * a.lddx + col, cols - col, u, a.nt);
  }
}
// Their weight gradients: a thread's V columns over the rows of the block's
// chunk (blocks.x chunks, blocks.y column tiles).
template <class T>
__global__ __launch_bounds__(kNormThreads) void k_norm_cols_wide(NormArgs a) {
  constexpr int V = Elem<T>::V;
  const int cols = a.cols, col = ((int)blockIdx.y * kNormThreads + (int)threadIdx.x) * V, n = cols - col;
  if (n <= 0) return;
  const RowsIn<T> xs{static_cast<const T*>(a.x), a.ldx, a.xq_in, a.xc_in};
  float dg[V] = {}, db[V] = {};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    float x[V], u[V];
    xs.load(row, col, cols, x);
    ld_piece<T>(static_cast<const T*>(a.dy) + row * a.ldy + col, n, u);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[i] += u[i] * ((x[i] - mean) * rstd);
      db[i] += u[i];
    }
  }
  float* out = a.part + (int64_t)blockIdx.x * 2 * cols + col;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) out[i] = dg[i], out[cols + i] = db[i];
}

// ------------------------------------------------------------ checkpoints
// Pieces of V values; consecutive threads take consecutive pieces of a row.
// Rows are padded to whole groups, so that a group never crosses a wave's
// 32 / V aligned lanes.
template <class T>
__global__ __launch_bounds__(256) void k_pack8(const T* x, int64_t ldx, int8_t* q, uint8_t* c, int64_t rows, int cols) {
  constexpr int V = Elem<T>::V;
  const int groups = (cols + kGroup - 1) / kGroup;
  const int64_t per = (int64_t)groups * (kGroup / V);
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  const int col = (int)(i - row * per) * V, n = row < rows ? cols - col : 0;
  float v[V];
  if (n > 0) ld_piece<T>(x + row * ldx + col, n, v);
  pack8_piece<V>(v, col, n, q + row * cols, c + row * groups);
}
template <class T>
__global__ __launch_bounds__(256) void k_unpack8(const int8_t* q, const uint8_t* c, T* x, int64_t ldx, int64_t rows,
                                                 int cols, bool nt) {
  constexpr int V = Elem<T>::V;
  const int groups = (cols + kGroup - 1) / kGroup;
  const int64_t per = (cols + V - 1) / V;
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  if (row >= rows) return;
  const int col = (int)(i - row * per) * V, n = cols - col;
  float v[V];
  get8(ld_raw8<V>(q + row * cols, c + row * groups, col, n), v);
  st_piece<T>(x + row * ldx + col, n, v, nt);
}

// ------------------------------------------------------------ host
// The narrowest arrangement that holds a row: lanes per row and pieces per
// lane; J = 0 past the registers.  The backward's are full past two pieces of
// bfloat16 in 512 lanes: four spilled 1 KB a lane, and reading the row again is
// faster (2,003 x 10,001 92 us against 209, 2,003 x 16,384 130 against 175, from 8
// bits 114 against 191); the forward's hold (2,003 x 16,384 29 against 39).
template <class T, bool BWD, class F>
auto norm_shape(int cols, F&& f) {
  constexpr int V = Elem<T>::V;
  const int pieces = (cols + V - 1) / V;
#define E3_SHAPE(L, J) if (pieces <= L * J) return f(std::integral_constant<int, L>{}, std::integral_constant<int, J>{})
  E3_SHAPE(8, 1);
  E3_SHAPE(16, 1);
  E3_SHAPE(32, 1);
  E3_SHAPE(64, 1);
  E3_SHAPE(64, 2);
  E3_SHAPE(64, 3);
  E3_SHAPE(256, 1);
  E3_SHAPE(256, 2);
  E3_SHAPE(256, 3);
  E3_SHAPE(512, 2);
  if constexpr (!BWD || V == 4) E3_SHAPE(512, 4);
#undef E3_SHAPE
  return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 0>{});
}

// Workgroups of the backward: two per CU, each at least one round of rows.
int norm_blocks(e3_dtype t, int64_t rows, int cols) {
  auto of = [&](auto L, auto J) {
    constexpr int l = decltype(L)::value, R = decltype(J)::value > 0 ? kNormBwdThreads<l> / l : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(512, (rows + R - 1) / R));
  };
  return t == E3_F32 ? norm_shape<float, true>(cols, of) : norm_shape<__bf16, true>(cols, of);
}

template <class T>
e3_status norm_fwd(const NormArgs& a, hipStream_t st) {
  return norm_shape<T, false>(a.cols, [&](auto L, auto J) -> e3_status {
    constexpr int l = decltype(L)::value, j = decltype(J)::value, R = kNormFwdThreads<l> / l;
    TimedLaunch t_("layer_norm_fwd", st);
    hipLaunchKernelGGL((k_norm_fwd<T, l, j>), grid_of((a.rows + R - 1) / R), dim3(kNormFwdThreads<l>), 0, st, a);
    E3_HIP(hipGetLastError());
    return E3_OK;
  });
}

template <class T>
e3_status norm_bwd(const NormArgs& a, hipStream_t st) {
  return norm_shape<T, true>(a.cols, [&](auto L, auto J) -> e3_status {
    constexpr int l = decltype(L)::value, j = decltype(J)::value;
    if constexpr (j > 0) {
      const bool fast = a.dx && a.nt && a.cols == l * j * Elem<T>::V;
      TimedLaunch t_(fast ? "layer_norm_bwd_stream" : "layer_norm_bwd", st);
      auto* k = a.x ? (fast ? k_norm_bwd<T, l, j, false, true> : k_norm_bwd<T, l, j, false, false>)
                    : (fast ? k_norm_bwd<T, l, j, true, true> : k_norm_bwd<T, l, j, true, false>);
      hipLaunchKernelGGL(k, dim3(a.blocks), dim3(kNormBwdThreads<l>), 0, st, a);
      E3_HIP(hipGetLastError());
    } else {
      if (a.dx) {
        TimedLaunch t_("layer_norm_bwd_wide", st);
        hipLaunchKernelGGL((k_norm_bwd_wide<T>), grid_of(a.rows), dim3(kNormThreads), 0, st, a);
        E3_HIP(hipGetLastError());
      }
      if (a.part) {
        TimedLaunch t_("layer_norm_bwd_cols", st);
        const int per = kNormThreads * Elem<T>::V;
        hipLaunchKernelGGL((k_norm_cols_wide<T>), dim3(a.blocks, (a.cols + per - 1) / per), dim3(kNormThreads), 0, st,
                           a);
        E3_HIP(hipGetLastError());
      }
    }
    return E3_OK;
  });
}

}  // namespace

extern "C" {

e3_status e3_pack8(e3_dtype dtype, const void* x, int64_t ldx, int8_t* q, uint8_t* c, int64_t rows, int64_t cols,
                   e3_stream stream) {
  if (!good_rows(dtype, rows, cols) || ldx < cols) return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!good_ptr(dtype, x) || !q || !c) return E3_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  TimedLaunch t_("pack8", st);
  const int64_t n = rows * ((cols + kGroup - 1) / kGroup) * kGroup;
  if (dtype == E3_F32)
    hipLaunchKernelGGL(k_pack8<float>, grid_of((n / 4 + 255) / 256), dim3(256), 0, st, static_cast<const float*>(x),
                       ldx, q, c, rows, (int)cols);
  else
    hipLaunchKernelGGL(k_pack8<__bf16>, grid_of((n / 8 + 255) / 256), dim3(256), 0, st, static_cast<const __bf16*>(x),
                       ldx, q, c, rows, (int)cols);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

e3_status e3_unpack8(e3_dtype dtype, const int8_t* q, const uint8_t* c, void* x, int64_t ldx, int64_t rows,
                     int64_t cols, e3_stream stream) {
  if (!good_rows(dtype, rows, cols) || ldx < cols) return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!good_ptr(dtype, x) || !q || !c) return E3_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  TimedLaunch t_("unpack8", st);
  if (dtype == E3_F32)
    hipLaunchKernelGGL(k_unpack8<float>, grid_of((rows * ((cols + 3) / 4) + 255) / 256), dim3(256), 0, st, q, c,
                       static_cast<float*>(x), ldx, rows, (int)cols, streams(dtype, rows, cols));
  else
    hipLaunchKernelGGL(k_unpack8<__bf16>, grid_of((rows * ((cols + 7) / 8) + 255) / 256), dim3(256), 0, st, q, c,
                       static_cast<__bf16*>(x), ldx, rows, (int)cols, streams(dtype, rows, cols));
  E3_HIP(hipGetLastError());
  return E3_OK;
}

e3_status e3_layer_norm_fwd(e3_dtype dtype, const void* x, int64_t ldx, const void* gamma, const void* beta, float eps,
                            void* y, int64_t ldy, float* mean, float* rstd, int8_t* xq, uint8_t* xc, int8_t* yq,
                            uint8_t* yc, int64_t rows, int64_t cols, e3_stream stream) {
  if (!good_rows(dtype, rows, cols) || ldx < cols || ldy < cols || !(eps >= 0.0f)) return E3_ERR_INVALID_ARG;
  if (!xq != !xc || !yq != !yc) return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!good_ptr(dtype, x) || !good_ptr(dtype, y) || misaligned(dtype, gamma) || misaligned(dtype, beta) ||
      misaligned(E3_F32, mean) || misaligned(E3_F32, rstd))
    return E3_ERR_INVALID_ARG;
  NormArgs a{};
  a.x = x, a.ldx = ldx, a.gamma = gamma, a.beta = beta, a.eps = eps, a.y = y, a.ldy = ldy, a.mean = mean;
  a.rstd = rstd, a.xq = xq, a.xc = xc, a.yq = yq, a.yc = yc, a.rows = rows, a.cols = (int)cols;
  a.nt = streams(dtype, rows, cols);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  return dtype == E3_F32 ? norm_fwd<float>(a, st) : norm_fwd<__bf16>(a, st);
}

e3_status e3_layer_norm_workspace_size(e3_dtype dtype, int64_t rows, int64_t cols, size_t* bwd_bytes) {
  if (!good_rows(dtype, rows, cols) || !bwd_bytes) return E3_ERR_INVALID_ARG;
  *bwd_bytes = rows == 0 ? 0 : ((size_t)norm_blocks(dtype, rows, (int)cols) * 2 * cols * sizeof(float) + 255) / 256 * 256;
  return E3_OK;
}

e3_status e3_layer_norm_bwd(e3_dtype dtype, const void* x, int64_t ldx, const int8_t* xq, const uint8_t* xc,
                            const void* gamma, const void* dy, int64_t lddy, const float* mean, const float* rstd,
                            void* dx, int64_t lddx, void* dgamma, void* dbeta, void* ws, size_t ws_bytes, int64_t rows,
                            int64_t cols, e3_stream stream) {
  if (!good_rows(dtype, rows, cols) || (x && ldx < cols) || lddy < cols || (dx && lddx < cols) || !xq != !xc)
    return E3_ERR_INVALID_ARG;
  if (rows > 0 && (!x == !xq || misaligned(dtype, x) || !good_ptr(dtype, dy) || !mean || !rstd ||
                   misaligned(E3_F32, mean) || misaligned(E3_F32, rstd)))
    return E3_ERR_INVALID_ARG;
  if (misaligned(dtype, gamma) || misaligned(dtype, dx) || misaligned(dtype, dgamma) || misaligned(dtype, dbeta))
    return E3_ERR_INVALID_ARG;
  const bool sums = dgamma || dbeta;
  size_t need = 0;
  (void)e3_layer_norm_workspace_size(dtype, rows, cols, &need);
  if (sums && ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (sums && need && (!ws || misaligned(E3_F32, ws))) return E3_ERR_INVALID_ARG;
  if (!dx && !sums) return E3_OK;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  NormArgs a{};
  a.x = x, a.ldx = ldx, a.xq_in = xq, a.xc_in = xc, a.gamma = gamma, a.dy = dy, a.ldy = lddy, a.dx = dx;
  a.lddx = lddx, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
  a.part = sums && rows ? static_cast<float*>(ws) : nullptr, a.rows = rows, a.cols = (int)cols;
  a.nt = streams(dtype, rows, cols);
  a.blocks = rows ? norm_blocks(dtype, rows, (int)cols) : 0;
  if (rows) {
    const e3_status s = dtype == E3_F32 ? norm_bwd<float>(a, st) : norm_bwd<__bf16>(a, st);
    if (s != E3_OK) return s;
  }
  if (!sums) return E3_OK;
  return column_sums(dtype, static_cast<const float*>(ws), a.blocks, 2 * cols, cols, 2 * cols, dgamma, dbeta, st);
}

}  // extern "C"
