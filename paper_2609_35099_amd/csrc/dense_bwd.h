// Dense layers: the backward, for the type of the including unit.
#pragma once
#include "dense.h"

namespace {

// The column sums of B alone, in the order in which the product sums them.
template <class J, int B>
__global__ __launch_bounds__((TileOf<J, B>::THREADS), (TileOf<J, B>::OCC)) void k_dense_sums(DenseArgs a) {
  using Tl = typename TileOf<J, B>::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  dense_block<J, Tl, TileOf<J, B>::BM, TileOf<J, B>::BN, true>(a, sh, block_id());
}
// Two products in one launch: the first `first` blocks take the first.
template <class J, class K, int B>
__global__ __launch_bounds__((TileOf<J, B>::THREADS), 2) void k_dense_two(DenseArgs a, DenseArgs b, int64_t first) {
  using Ta = typename TileOf<J, B>::type;
  using Tb = typename TileOf<K, B>::type;
  static_assert(Ta::THREADS == Tb::THREADS);
  __shared__ __align__(16) union {
    typename Ta::Shared a;
    typename Tb::Shared b;
  } sh;
  const int64_t u = block_id();
  if (u < first) dense_block<J, Ta, B, B>(a, sh.a, u);
  else dense_block<K, Tb, B, B>(b, sh.b, u - first);
}

// dz = dy act'(z) in the type of dy (a bfloat16 dz is an operand of the matrix
// instructions, which take no more bits: Kind says what that costs), and the column sums of its unrounded
// values over the block's rows, for layers whose products would form dz too often
// themselves (forms_dz).  Either output may be null.
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

// Layers of which a matrix is shorter than a piece, and not many rows: a wave per
// value of dx, dW and db, whose lanes take every 64th term.
template <class T>
__global__ __launch_bounds__(256) void k_dense_bwd_tiny(RowsIn<T> x, const T* W, RowsIn<T> z, int act, const T* dy,
                                                        int64_t lddy, T* dx, int64_t lddx, T* dW, T* db, int64_t M,
                                                        int K, int N) {
  const int l = threadIdx.x % kWave;
  int64_t u = block_id() * 4 + threadIdx.x / kWave;
  auto dz = [&](int64_t m, int n) {
    const float v = Elem<T>::one(dy[m * lddy + n]);
    return act == E3_ACT_NONE ? v : v * act_grad(act, z.value(m, n, N));
  };
  float v = 0.0f;
  T* out;
  if (u < M * K) {
    if (!dx) return;
    const int64_t m = u / K, k = u % K;
    for (int n = l; n < N; n += kWave) v = fmaf(Elem<T>::round(dz(m, n)), Elem<T>::one(W[k * N + n]), v);
    out = dx + m * lddx + k;
  } else if ((u -= M * K) < (int64_t)K * N) {
    if (!dW) return;
    const int k = (int)(u / N), n = (int)(u % N);
    for (int64_t m = l; m < M; m += kWave) v = fmaf(x.value(m, k, K), Elem<T>::round(dz(m, n)), v);
    out = dW + u;
  } else {
    u -= (int64_t)K * N;
    if (!db || u >= N) return;
    for (int64_t m = l; m < M; m += kWave) v += dz(m, (int)u);
    out = db + u;
  }
  v = sum_lanes<kWave>(v);
  if (l == 0) *out = (T)v;
}

// A W shorter than a piece, so that whole pieces can be read.
template <class T>
__global__ __launch_bounds__(kWave) void k_dense_short(const T* W, int n, T* out) {
  const int i = threadIdx.x;
  if (i < Elem<T>::V) out[i] = i < n ? W[i] : (T)0.0f;
}

// ------------------------------------------------------------ host
// dx and dW (FLY: and db) of a layer whose operand dz is of kind KD and x of KX.
template <class T, Kind KD, Kind KX, bool FLY>
e3_status dense_bwd_products(DenseArgs x, DenseArgs w, float* part, hipStream_t st) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  using JX = Job<T, kAlong, kAlong, KD, kFull, false>;
  using JW = Job<T, kAcross, kAcross, KX, KD, FLY>;
  const bool dx = x.y, dw = w.y, db = w.sums;
  const Cut cx = dense_cut(t, x.rows, x.cols, x.red, kDx), cw = dense_cut(t, w.rows, w.cols, w.red, kDw);
  const bool along = panel<T>(x.rows, x.cols, x.red);
  set_cut(x, cx, part);
  set_cut(w, cw, part + cut_bytes(cx, x.rows, x.cols) / sizeof(float), w.cols);
  e3_status s = E3_OK;
  if (dx && dw && !along && cx.tile == 64 && cw.tile == 64) {
    TimedLaunch t_("dense_bwd_both", st);
    const int64_t first = cx.tiles * cx.splits;
    hipLaunchKernelGGL((k_dense_two<JX, JW, 64>), grid_of(first + cw.tiles * cw.splits), dim3(256), 0, st, x, w, first);
    E3_HIP(hipGetLastError());
  } else {
    if (dx) s = along ? dense_panel<JX>(x, kNamesDx, st) : dense_launch<JX>(x, cx, kNamesDx, st);
    if (s == E3_OK && dw) s = dense_launch<JW>(w, cw, kNamesDw, st);
  }
  if constexpr (FLY && KX == kFull) {
    if (s == E3_OK && db && !dw) {
      TimedLaunch t_(kNamesDb.tile(cw.tile), st);
      const dim3 grid = grid_of((w.cols + cw.tile - 1) / cw.tile * (int64_t)cw.splits);
      auto go = [&](auto B) {
        constexpr int b = decltype(B)::value;
        hipLaunchKernelGGL((k_dense_sums<JW, b>), grid, dim3(TileOf<JW, b>::THREADS), 0, st, w);
      };
      if (cw.tile == 64) go(std::integral_constant<int, 64>{});
      else if (cw.tile == 128) go(std::integral_constant<int, 128>{});
      else if constexpr (sizeof(T) == 2 && KD != kGradPacked) go(std::integral_constant<int, 256>{});
      E3_HIP(hipGetLastError());
    }
  }
  if (s == E3_OK && dx && !along && cx.splits > 1) s = dense_join<T>(x, st);
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
  constexpr int V = Elem<T>::V;
  // x or dy shorter than a piece; a short W (copied to a whole piece below) where its
  // launches would cost more than the wave's long sums: float32 silu, in one launch
  // against tiles, us: 300 x 1 x 3 15 against 20, 6,000 20 and 20, 10,003 32 against
  // 20, 1,000,003 5,410 against 235.
  if (M * N < V || M * K < V || (K * N < V && M <= 4096)) {
    TimedLaunch t_("dense_bwd_tiny", st);
    const int64_t outs = M * K + K * N + N;
    hipLaunchKernelGGL(k_dense_bwd_tiny<T>, grid_of((outs + 3) / 4), dim3(256), 0, st, x, W, z, act, dy, lddy, dx, lddx,
                       dW, db, M, (int)K, (int)N);
    E3_HIP(hipGetLastError());
    return E3_OK;
  }
  const DenseBwdWs w = dense_bwd_ws(t, M, K, N);
  const bool fly = forms_dz(t, M, K, N, act != E3_ACT_NONE && z.q);
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
  int64_t total = K * N;
  if (dx && total < V) {
    TimedLaunch t_("dense_short", st);
    T* copy = reinterpret_cast<T*>(ws + w.dz + w.db + w.part);
    hipLaunchKernelGGL(k_dense_short<T>, dim3(1), dim3(kWave), 0, st, W, (int)total, copy);
    E3_HIP(hipGetLastError());
    W = copy, total = V;
  }
  DenseArgs ax{}, aw{};
  const int64_t ldd = own ? N : lddy, ldz = z.x ? z.ld : N, ldx = x.x ? x.ld : K;
  const Side d{own ? dz : dy, ldd, nullptr, nullptr, 0, (M - 1) * ldd + N};
  const Side pre{z.x, ldz, z.q, z.c, (N + kGroup - 1) / kGroup, (M - 1) * ldz + N};
  ax.a = d, ax.b = {W, N, nullptr, nullptr, 0, total}, ax.pre = pre, ax.grad_act = act, ax.rows = M, ax.cols = (int)K, ax.red = N;
  ax.y = dx, ax.ldy = lddx, ax.nt = streams(t, M, K);
  aw.a = {x.x, ldx, x.q, x.c, (K + kGroup - 1) / kGroup, (M - 1) * ldx + K}, aw.b = d, aw.pre = pre, aw.grad_act = act;
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
e3_status dense_bwd_call(const DenseBwdCall& c) {
  return dense_bwd<T>({static_cast<const T*>(c.x), c.ldx, c.xq, c.xc}, static_cast<const T*>(c.W),
                      {static_cast<const T*>(c.z), c.ldz, c.zq, c.zc}, c.act, static_cast<const T*>(c.dy), c.lddy,
                      static_cast<T*>(c.dx), c.lddx, static_cast<T*>(c.dW), static_cast<T*>(c.db), c.ws, c.M, c.K, c.N,
                      c.st);
}

}  // namespace
