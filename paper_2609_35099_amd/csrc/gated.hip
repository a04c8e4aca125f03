// e3mi: gated dense layers: the C entry points and the backward's way to dz.  The
// forward is in gated.h (a unit per type), the backward's products are the dense
// layers' (dense_bwd.h).
#include "gated.h"

namespace {

// g or u, in full or packed.
template <class T>
struct Halves {
  RowsIn<T> g, u;
};

// dz in the type of dy (bfloat16: an operand of the matrix instructions, which take no
// more bits), and the column sums of its unrounded values over the block's rows.
// Either output may be null.  Bound by memory: reads dy, g and u, writes two halves.
template <class T>
__global__ __launch_bounds__(256) void k_gated_dz(Halves<T> z, int act, const T* dy, int64_t lddy, T* dz, float* part,
                                                  int64_t rows, int cols, int64_t per) {
  constexpr int V = Elem<T>::V, CL = 16, RL = 256 / CL;
  __shared__ float s[RL][CL * V];
  const int cl = threadIdx.x % CL, rl = threadIdx.x / CL;
  const int col = ((int)blockIdx.y * CL + cl) * V, n = cols - col;
  const int64_t row0 = blockIdx.x * per, row1 = row0 + per < rows ? row0 + per : rows;
  float sum[2][V] = {};
  for (int64_t row = row0 + rl; row < row1; row += RL) {
    float d[V], g[V], u[V], e[V];
    ld_piece<T>(dy + row * lddy + col, n, d);
    z.g.load(row, col, cols, g);
    z.u.load(row, col, cols, u);
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = i < n ? u[i] * d[i] : 0.0f, e[i] = i < n ? g[i] : 0.0f;
    act_grad_piece(act, g, u);
    act_piece(act, e);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      e[i] = i < n ? e[i] * d[i] : 0.0f;
      u[i] = i < n ? u[i] : 0.0f;
      sum[0][i] += u[i], sum[1][i] += e[i];
    }
    if (dz) {
      T* to = dz + row * 2 * cols + col;
      st_piece<T>(to, n, u);
      st_piece<T>(to + cols, n, e);
    }
  }
  if (!part) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) s[rl][cl * V + i] = sum[h][i];
    __syncthreads();
    for (int i = threadIdx.x; i < CL * V; i += 256) {
      const int c = (int)blockIdx.y * CL * V + i;
      if (c >= cols) continue;
      float v = 0.0f;
#pragma unroll
      for (int r = 0; r < RL; ++r) v += s[r][i];
      part[((int64_t)blockIdx.x * 2 + h) * cols + c] = v;
    }
  }
}

struct GatedBwdWs {
  size_t dz, db, products, total;
  int64_t blocks, rows;  // of the pass that forms dz
};
GatedBwdWs gated_bwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  GatedBwdWs w{};
  if (M == 0) return w;
  // 4,096 workgroups with the column tiles: more would leave more partial sums of db
  const int64_t tiles = (N + 16 * (t == E3_F32 ? 4 : 8) - 1) / (16 * (t == E3_F32 ? 4 : 8));
  w.blocks = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512, std::max<int64_t>(64, 4096 / tiles)), (M + 63) / 64));
  w.rows = (M + w.blocks - 1) / w.blocks;
  w.dz = up256((size_t)M * 2 * N * (t == E3_F32 ? 4 : 2));
  w.db = up256((size_t)w.blocks * 2 * N * 4);
  w.products = dense_bwd_ws(t, M, K, 2 * N, true).total;
  w.total = w.dz + w.db + w.products;
  if (gated_fused(M, K, N))  // from z in full or packed
    w.total = std::max(w.total, up256((size_t)gated_fused_groups(t, M, N) * (K * 2 * N + 2 * N) * 4));
  return w;
}

template <class T>
e3_status gated_bwd(const GatedCall& c) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  if (gated_fused(c.M, c.K, c.N) && c.z_in) return t == E3_F32 ? gated_bwd_fused_f32(c) : gated_bwd_fused_bf16(c);
  const GatedBwdWs w = gated_bwd_ws(t, c.M, c.K, c.N);
  T* dz = reinterpret_cast<T*>(c.ws);
  float* part = reinterpret_cast<float*>(c.ws + w.dz);
  const bool products = c.dx || c.dW;
  {
    TimedLaunch t_("gated_dz", c.st);
    const T* z = static_cast<const T*>(c.z_in);
    const Halves<T> halves{{z, c.ldz, c.gq_in, c.gc_in}, {z ? z + c.N : nullptr, c.ldz, c.uq_in, c.uc_in}};
    const int per = 16 * Elem<T>::V;
    hipLaunchKernelGGL(k_gated_dz<T>, dim3((unsigned)w.blocks, (unsigned)((c.N + per - 1) / per)), dim3(256), 0, c.st,
                       halves, c.act, static_cast<const T*>(c.dy), c.lddy, products ? dz : nullptr, c.db ? part : nullptr,
                       c.M, (int)c.N, w.rows);
    E3_HIP(hipGetLastError());
  }
  if (c.db) {
    const e3_status s = column_sums(t, part, (int)w.blocks, 2 * c.N, 2 * c.N, 2 * c.N, c.db, nullptr, c.st);
    if (s != E3_OK) return s;
  }
  if (!products) return E3_OK;
  const DenseBwdCall d{c.dtype, c.x,   c.W,     nullptr, dz,     c.xq,   nullptr, c.xc, nullptr, c.dx, c.dW,        nullptr,
                       c.ws + w.dz + w.db, c.ldx, 0, 2 * c.N, c.lddx, c.M, c.K, 2 * c.N, E3_ACT_NONE, c.st, true};
  return t == E3_F32 ? dense_bwd_f32(d) : dense_bwd_bf16(d);
}

bool good_gated(e3_dtype t, int64_t M, int64_t K, int64_t N, e3_act act) {
  return good_rows(t, M, K) && N >= 1 && 2 * N <= kMaxCols && act >= E3_ACT_NONE && act <= E3_ACT_GELU;
}
template <class T>
__global__ __launch_bounds__(256) void k_gated_zero(T* p, int64_t n) {
  const int64_t i = block_id() * 256 + threadIdx.x;
  if (i < n) p[i] = (T)0.0f;
}
e3_status gated_zeros(e3_dtype t, void* p, int64_t n, hipStream_t st) {
  if (!p) return E3_OK;
  TimedLaunch t_("gated_zero", st);
  if (t == E3_F32)
    hipLaunchKernelGGL(k_gated_zero<float>, grid_of((n + 255) / 256), dim3(256), 0, st, static_cast<float*>(p), n);
  else
    hipLaunchKernelGGL(k_gated_zero<__bf16>, grid_of((n + 255) / 256), dim3(256), 0, st, static_cast<__bf16*>(p), n);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

}  // namespace

extern "C" {

e3_status e3_gated_workspace_size(e3_dtype dtype, int64_t M, int64_t K, int64_t N, size_t* fwd_bytes,
                                  size_t* bwd_bytes) {
  if (!good_gated(dtype, M, K, N, E3_ACT_NONE) || !fwd_bytes || !bwd_bytes) return E3_ERR_INVALID_ARG;
  *fwd_bytes = gated_fwd_ws(dtype, M, K, N);
  *bwd_bytes = gated_bwd_ws(dtype, M, K, N).total;
  return E3_OK;
}

e3_status e3_gated_fwd(e3_dtype dtype, const void* x, int64_t ldx, const void* W, const void* bias, e3_act act, void* y,
                       int64_t ldy, void* z, int64_t ldz, int8_t* gq, uint8_t* gc, int8_t* uq, uint8_t* uc, int8_t* yq,
                       uint8_t* yc, void* ws, size_t ws_bytes, int64_t M, int64_t K, int64_t N, e3_stream stream) {
  if (!good_gated(dtype, M, K, N, act) || ldx < K || ldy < N || (z && ldz < 2 * N) || !gq != !gc || !uq != !uc ||
      !gq != !uq || !yq != !yc)
    return E3_ERR_INVALID_ARG;
  if (M == 0) return E3_OK;
  if (!good_ptr(dtype, x) || !good_ptr(dtype, W) || !good_ptr(dtype, y) || misaligned(dtype, bias) || misaligned(dtype, z))
    return E3_ERR_INVALID_ARG;
  const size_t need = gated_fwd_ws(dtype, M, K, N);
  if (ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (need && (!ws || misaligned(E3_F32, ws))) return E3_ERR_INVALID_ARG;
  GatedCall c{};
  c.dtype = dtype, c.x = x, c.W = W, c.bias = bias, c.ldx = ldx, c.act = act, c.y = y, c.z = z, c.ldy = ldy, c.ldz = ldz;
  c.gq = gq, c.gc = gc, c.uq = uq, c.uc = uc, c.yq = yq, c.yc = yc, c.ws = static_cast<char*>(ws), c.M = M, c.K = K;
  c.N = N, c.st = reinterpret_cast<hipStream_t>(stream);
  return dtype == E3_F32 ? gated_fwd_f32(c) : gated_fwd_bf16(c);
}

e3_status e3_gated_bwd(e3_dtype dtype, const void* x, int64_t ldx, const int8_t* xq, const uint8_t* xc, const void* W,
                       const void* z, int64_t ldz, const int8_t* gq, const uint8_t* gc, const int8_t* uq,
                       const uint8_t* uc, e3_act act, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dW,
                       void* db, void* ws, size_t ws_bytes, int64_t M, int64_t K, int64_t N, e3_stream stream) {
  if (!good_gated(dtype, M, K, N, act) || (x && ldx < K) || (z && ldz < 2 * N) || lddy < N || (dx && lddx < K) ||
      !xq != !xc || !gq != !gc || !uq != !uc || !gq != !uq)
    return E3_ERR_INVALID_ARG;
  if (misaligned(dtype, x) || misaligned(dtype, W) || misaligned(dtype, z) || misaligned(dtype, dx) ||
      misaligned(dtype, dW) || misaligned(dtype, db))
    return E3_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (M == 0) {
    const e3_status s = gated_zeros(dtype, dW, K * 2 * N, st);
    return s != E3_OK ? s : gated_zeros(dtype, db, 2 * N, st);
  }
  if (!good_ptr(dtype, dy) || (dx && !W) || (dW && !x == !xq) || (x && xq) || !z == !gq) return E3_ERR_INVALID_ARG;
  if (!dx && !dW && !db) return E3_OK;
  const size_t need = gated_bwd_ws(dtype, M, K, N).total;
  if (ws_bytes < need) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) & 15u)) return E3_ERR_INVALID_ARG;
  GatedCall c{};
  c.dtype = dtype, c.x = x, c.W = W, c.ldx = ldx, c.act = act, c.z_in = z, c.ldz = ldz, c.dy = dy, c.lddy = lddy;
  c.xq = xq, c.xc = xc, c.gq_in = gq, c.gc_in = gc, c.uq_in = uq, c.uc_in = uc, c.dx = dx, c.lddx = lddx, c.dW = dW;
  c.db = db, c.ws = static_cast<char*>(ws), c.M = M, c.K = K, c.N = N, c.st = st;
  return dtype == E3_F32 ? gated_bwd<float>(c) : gated_bwd<__bf16>(c);
}

}  // extern "C"
