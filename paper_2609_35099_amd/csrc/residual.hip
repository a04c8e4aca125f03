// e3mi: dropout, and what stands between two blocks of a residual network: the
// norm after a block, dropout, gate, residual scale, the sum and the norm before
// the next block, in one pass, forward and backward.
//
//   s = r + scale gate drop(N1(h)),  y = N2(s)
//   N(x) = n gamma (+ beta),  n = x rstd or (x - mean) rstd
// backward, with a2 = dy gamma2 and a1 = t gate gamma1:
//   d  = ds + rstd2 (a2 - n2 mean(a2 n2) [- mean(a2)])        (dr = d)
//   t  = scale drop(d),  dgate = t N1(h) where it was kept
//   dh = rstd1 (a1 - n1 mean(a1 n1) [- mean(a1)])
//   dgamma2 = sum dy n2, dbeta2 = sum dy, dgamma1 = sum t gate n1, dbeta1 = sum t gate
//
// Rows are read once, kept in registers and written once.  From 32 float32 or 64 bfloat16
// columns to the registers' end, whole pieces are bound by memory (and the mask by its
// multiplications, of which half as many fit beside a bfloat16 read and write): bfloat16
// 65,536 x 1,024, rms: forward 103 us (5.2 TB/s), backward 155 (the rate of a copy of its
// bytes), dropout of it 53 to 65; float32 100,003 x 515 with layer norms and a gate by row
// and column, backward 345 (a copy 326).  N2 sees the float32 sum, not the s that is stored.
// L lanes share a row, J 16-byte pieces each; rows past the registers are read
// again for each pass.
// Not so bound, us and a copy of the bytes (rms, both norms, a row gate, dropout; forward,
// backward): narrow rows, by rounds of latency, as eight lanes share a row at least and a CU
// has 64 of them in the backward, 600,000 x 16 float32 38 of 30 and 72 of 45, bfloat16 46 of
// 15 and 93 of 23, 1,000,000 x 8 55 of 25 and 107 of 38, 73 of 13 and 141 of 19; bfloat16 rows
// of odd lengths, whose last pieces go value by value, 100,003 x 515 135 of 81 and 351 of 121;
// rows past the registers, by reading them two to three times, 2,001 x 10,001 float32 87 of
// 63 and 229 of 94, bfloat16 61 of 31 and 204 of 47.
#include "drop.h"

namespace {

struct ResArgs {
  const void *h, *res, *gate, *g1, *b1, *g2, *b2;
  void *s, *y;
  float *mean1, *rstd1, *mean2, *rstd2;
  // backward (s_in: the forward's s)
  const void *s_in, *dy, *ds;
  void *dr, *dh, *dgate;
  float* part;   // [blocks][slots][cols]: partial sums over rows
  float* means;  // [rows][2]: the two means of N2's backward, of rows past the registers
  int64_t ldh, ldr, ldg, lds, ldy, ldd, lddr, lddh, lddg, rows;
  int cols, blocks;
  int slot[5];   // of dgamma1, dbeta1, dgamma2, dbeta2, dgate in part (-1: not wanted)
  int slots;
  Drop drop;
  float scale, eps;
  bool post, pre, nt;
};
enum { kDg1, kDb1, kDg2, kDb2, kDgate };

// Sums over the L lanes of a row: part of a wave, or the whole workgroup (then
// every thread calls it; `s` holds N values per wave).
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* s) {
  if constexpr (L <= kWave) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sum_lanes<L>(v[k]);
  } else {
    constexpr int W = L / kWave;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = sum_lanes<kWave>(v[k]);
      if (threadIdx.x % kWave == 0) s[k * W + threadIdx.x / kWave] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) v[k] += s[k * W + w];
    }
    __syncthreads();
  }
}

// n = (x - mean) rstd + shift.  The mean is a float32, which is off by up to 2^-24
// of itself; shift takes the mean of the deviations from it, so that this stays out
// of n (and stored() is the corrected mean).
struct Stats {
  float mean, rstd, shift, stored;
  __device__ __forceinline__ float operator()(float x) const { return fmaf(x - mean, rstd, shift); }
};
// Those of a row: each(f) calls f(value) for the lane's values in the row.
template <int L, bool LAYER, class Each>
__device__ __forceinline__ Stats row_stats(Each&& each, float cols, float eps, float* s) {
  Stats r{};
  if constexpr (LAYER) {
    float m[1] = {};
    each([&](float x) { m[0] += x; });
    row_sums<L>(m, s);
    r.mean = m[0] / cols;
    float q[2] = {};
    each([&](float x) {
      const float d = x - r.mean;
      q[0] += d;
      q[1] = fmaf(d, d, q[1]);
    });
    row_sums<L>(q, s);
    const float dev = q[0] / cols;
    float var = fmaf(-dev, dev, q[1] / cols);
    if (var < 0.0f) var = 0.0f;  // (a NaN stays)
    r.rstd = 1.0f / sqrtf(var + eps);
    r.shift = -dev * r.rstd;
    r.stored = r.mean + dev;
  } else {
    float q[1] = {};
    each([&](float x) { q[0] = fmaf(x, x, q[0]); });
    row_sums<L>(q, s);
    r.rstd = 1.0f / sqrtf(q[0] / cols + eps);
  }
  return r;
}
// gamma (1) or beta (0) at a piece.
template <class T>
__device__ __forceinline__ void ld_weight(const void* p, int col, int n, float none, float (&v)[Elem<T>::V]) {
  if (p) {
    ld_piece<T>(static_cast<const T*>(p) + col, n, v);
  } else {
#pragma unroll
    for (int i = 0; i < Elem<T>::V; ++i) v[i] = none;
  }
}
// v to its norm; zero past the row's end.
template <class T>
__device__ __forceinline__ void norm_piece(const Stats& st, const void* gamma, const void* beta, int col, int n,
                                           float (&v)[Elem<T>::V]) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V;
  float g[V], b[V];
  ld_weight<T>(gamma, col, n, 1.0f, g);
  ld_weight<T>(beta, col, n, 0.0f, b);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = i < n ? fmaf(st(v[i]), g[i], b[i]) : 0.0f;
}
// The way of a piece of N1(h) to the sum.
template <int V>
__device__ __forceinline__ void to_sum(const ResArgs& a, const Dropper& drop, int64_t row, int col, const float (&gate)[V],
                                       const float (&res)[V], float (&v)[V]) {
#pragma clang fp contract(off)
  if (drop.t) {
    const unsigned keep = drop.kept<V>(row, col);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = keep >> i & 1 ? v[i] * a.drop.grow : 0.0f;
  }
  if (a.gate)
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= gate[i];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = a.res ? fmaf(a.scale, v[i], res[i]) : a.scale * v[i];
}

template <int L>
constexpr int kResThreads = L <= kWave ? 256 : L;
template <class T, int L, int J, bool LAYER>
__global__ __launch_bounds__(kResThreads<L>) void k_res_fwd(ResArgs a) {
  constexpr int V = Elem<T>::V, R = kResThreads<L> / L;
  __shared__ float sh[2 * kResThreads<L> / kWave];
  const int lane = threadIdx.x % L, cols = a.cols;
  const int64_t row = block_id() * R + threadIdx.x / L;
  if (row >= a.rows) return;  // whole rows leave: no lane of another row's group
  const Dropper drop(a.drop);
  typename Elem<T>::vec hr[J], rr[J], gr[J];
  const T* h = static_cast<const T*>(a.h) + row * a.ldh;
  const T* res = static_cast<const T*>(a.res) + row * a.ldr;
  const T* gate = static_cast<const T*>(a.gate) + row * a.ldg;
#pragma unroll
  for (int j = 0; j < J; ++j) hr[j] = ld_raw<T>(h + (j * L + lane) * V, cols - (j * L + lane) * V);
  if (a.res)
#pragma unroll
    for (int j = 0; j < J; ++j) rr[j] = ld_raw<T>(res + (j * L + lane) * V, cols - (j * L + lane) * V);
  if (a.gate)
#pragma unroll
    for (int j = 0; j < J; ++j) gr[j] = ld_raw<T>(gate + (j * L + lane) * V, cols - (j * L + lane) * V);
  float v[J][V];
#pragma unroll
  for (int j = 0; j < J; ++j) Elem<T>::get(hr[j], v[j]);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < cols - (j * L + lane) * V) f(v[j][i]);
  };
  if (a.post) {
    const Stats st = row_stats<L, LAYER>(each, (float)cols, a.eps, sh);
    if (lane == 0) {
      if (LAYER && a.mean1) a.mean1[row] = st.stored;
      if (a.rstd1) a.rstd1[row] = st.rstd;
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
      norm_piece<T>(st, a.g1, a.b1, (j * L + lane) * V, cols - (j * L + lane) * V, v[j]);
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int col = (j * L + lane) * V, n = cols - col;
    float g[V] = {}, r[V] = {};
    if (a.gate) Elem<T>::get(gr[j], g);
    if (a.res) Elem<T>::get(rr[j], r);
    to_sum<V>(a, drop, row, col, g, r, v[j]);
    if (a.s) st_piece<T>(static_cast<T*>(a.s) + row * a.lds + col, n, v[j], a.nt);
  }
  if (!a.pre) return;
  const Stats st = row_stats<L, LAYER>(each, (float)cols, a.eps, sh);
  if (lane == 0) {
    if (LAYER && a.mean2) a.mean2[row] = st.stored;
    if (a.rstd2) a.rstd2[row] = st.rstd;
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int col = (j * L + lane) * V, n = cols - col;
    norm_piece<T>(st, a.g2, a.b2, col, n, v[j]);
    st_piece<T>(static_cast<T*>(a.y) + row * a.ldy + col, n, v[j], a.nt);
  }
}

// Rows past the registers: a workgroup a row, read again for each pass.  s may be r:
// both are read by the thread that writes s, in the last pass, before it does.
template <class T, bool LAYER>
__global__ __launch_bounds__(512) void k_res_fwd_wide(ResArgs a) {
  constexpr int V = Elem<T>::V, L = 512;
  __shared__ float sh[2 * L / kWave];
  const int lane = threadIdx.x, cols = a.cols;
  const int64_t row = block_id();
  if (row >= a.rows) return;
  const Dropper drop(a.drop);
  const T* h = static_cast<const T*>(a.h) + row * a.ldh;
  const T* res = static_cast<const T*>(a.res) + row * a.ldr;
  const T* gate = static_cast<const T*>(a.gate) + row * a.ldg;
  Stats first{}, last{};
  if (a.post) {
    first = row_stats<L, LAYER>(
        [&](auto&& f) {
          for (int col = lane * V; col < cols; col += L * V) {
            float v[V];
            ld_piece<T>(h + col, cols - col, v);
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (i < cols - col) f(v[i]);
          }
        },
        (float)cols, a.eps, sh);
    if (lane == 0) {
      if (LAYER && a.mean1) a.mean1[row] = first.stored;
      if (a.rstd1) a.rstd1[row] = first.rstd;
    }
  }
  auto sum = [&](int col, float(&v)[V]) {
    const int n = cols - col;
    float g[V] = {}, r[V] = {};
    ld_piece<T>(h + col, n, v);
    if (a.gate) ld_piece<T>(gate + col, n, g);
    if (a.res) ld_piece<T>(res + col, n, r);
    if (a.post) norm_piece<T>(first, a.g1, a.b1, col, n, v);
    to_sum<V>(a, drop, row, col, g, r, v);
  };
  if (a.pre) {
    last = row_stats<L, LAYER>(
        [&](auto&& f) {
          for (int col = lane * V; col < cols; col += L * V) {
            float v[V];
            sum(col, v);
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (i < cols - col) f(v[i]);
          }
        },
        (float)cols, a.eps, sh);
    if (lane == 0) {
      if (LAYER && a.mean2) a.mean2[row] = last.stored;
      if (a.rstd2) a.rstd2[row] = last.rstd;
    }
  }
  for (int col = lane * V; col < cols; col += L * V) {
    float v[V];
    sum(col, v);
    if (a.s) st_piece<T>(static_cast<T*>(a.s) + row * a.lds + col, cols - col, v, a.nt);
    if (!a.pre) continue;
    norm_piece<T>(last, a.g2, a.b2, col, cols - col, v);
    st_piece<T>(static_cast<T*>(a.y) + row * a.ldy + col, cols - col, v, a.nt);
  }
}

// ------------------------------------------------------------ backward
// What is fused into sums is written out, so that every instance rounds alike.
// N2's part of a piece: x becomes n2, u (dy) becomes a2.
template <int V, bool LAYER>
__device__ __forceinline__ void second_piece(float mean, float rstd, const float (&g)[V], int n, float (&x)[V],
                                             float (&u)[V], float (&dg)[V], float (&db)[V], float (&c)[2]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < V; ++i) {
    // columns past the end have dy = 0: x there must not turn them into NaN
    x[i] = i < n ? (LAYER ? (x[i] - mean) * rstd : x[i] * rstd) : 0.0f;
    dg[i] = fmaf(u[i], x[i], dg[i]);
    if (LAYER) db[i] += u[i];
    u[i] *= g[i];
    c[0] = fmaf(u[i], x[i], c[0]);
    if (LAYER) c[1] += u[i];
  }
}
// The cotangent of a norm's input.
template <bool LAYER>
__device__ __forceinline__ float through(float rstd, float a, float n, const float (&c)[2]) {
  return rstd * fmaf(-n, c[0], LAYER ? a - c[1] : a);
}
// The row's means of what c holds the lane's sums of.
template <int L, bool LAYER>
__device__ __forceinline__ void row_means(float (&c)[2], float cols, float* s) {
  if constexpr (LAYER) {
    row_sums<L>(c, s);
    c[1] /= cols;
  } else {
    float one[1] = {c[0]};
    row_sums<L>(one, s);
    c[0] = one[0];
  }
  c[0] /= cols;
}
// N1's part of a piece: d becomes t gate, x (h) becomes n1, and dgate's terms come out.
template <int V, bool LAYER>
__device__ __forceinline__ void first_piece(const ResArgs& a, bool post, const Dropper& drop, int64_t row, int col, int n,
                                            float mean, float rstd, const float (&g1)[V], const float (&b1)[V], const float (&gate)[V],
                                            float (&x)[V], float (&d)[V], float (&dgate)[V]) {
#pragma clang fp contract(off)
  unsigned keep = ~0u;
  const float k = drop.t ? a.scale * a.drop.grow : a.scale;
  if (drop.t) keep = drop.kept<V>(row, col);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool in = i < n && (keep >> i & 1);
    d[i] = in ? d[i] * k : 0.0f;
    float o = x[i];
    if (post) {
      x[i] = i < n ? (LAYER ? (x[i] - mean) * rstd : x[i] * rstd) : 0.0f;
      o = fmaf(x[i], g1[i], b1[i]);
    }
    dgate[i] = in ? d[i] * o : 0.0f;
    if (a.gate) d[i] *= gate[i];
  }
}

// dr, dh, dgate of rows, and per workgroup the sums over its rows (rows blockIdx.x R
// + i, then every gridDim.x R).  The next row's pieces are in flight while a row is
// worked on; weights are kept in registers (their loads, issued after the next row's,
// would wait for those).
// FAST: both norms, ds, dr and dh, whole pieces, outputs that stream: no branch around
// a load or store, so that the wait for the next row leaves this one's stores in flight.
template <class T, int L, int J, bool LAYER, bool POST, bool FAST>
__global__ __launch_bounds__(kResThreads<L>, FAST ? 2 : 1) void k_res_bwd(ResArgs a) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V, NT = kResThreads<L>, R = NT / L;
  using Vec = typename Elem<T>::vec;
  __shared__ float sh[2 * NT / kWave];
  __shared__ float fold[R > 1 ? NT * V : 1];
  const int lane = threadIdx.x % L, cols = a.cols;
  const Dropper drop(a.drop);
  const float width = (float)cols;
  static_assert(POST || !FAST);
  constexpr bool post = POST;
  const bool pre = FAST || a.pre, full = !FAST && a.gate && a.ldg;
  float dg1[J][V] = {}, db1[J][V] = {}, dg2[J][V] = {}, db2[J][V] = {}, dgt[J][V] = {};
  const int64_t stride = (int64_t)gridDim.x * R;
  Vec hr[J], sr[J], yr[J], dr[J], gr[J], w1[J], w2[J], o1[J];
  float m1 = 0.0f, r1 = 0.0f, m2 = 0.0f, r2 = 0.0f;
  auto col_of = [&](int j) { return (j * L + lane) * V; };
  auto left = [&](int j) { return FAST ? V : cols - col_of(j); };
  auto rows_of = [&](const void* p, int64_t ld, int64_t r, Vec(&to)[J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) to[j] = ld_raw<T>(static_cast<const T*>(p) + r * ld + col_of(j), left(j));
  };
  auto weights = [&](const void* p, float none, Vec(&to)[J]) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = none;
#pragma unroll
    for (int j = 0; j < J; ++j) to[j] = Elem<T>::put(v);
    if (p) rows_of(p, 0, 0, to);
  };
#pragma unroll
  for (int j = 0; j < J; ++j) hr[j] = sr[j] = yr[j] = dr[j] = gr[j] = Vec{};
  weights(a.g1, 1.0f, w1), weights(a.g2, 1.0f, w2), weights(a.b1, 0.0f, o1);
  if (a.gate && !full) rows_of(a.gate, 0, 0, gr);
  auto load = [&](int64_t r) {
    if (r >= a.rows) r = a.rows - 1;
    if (pre) {
      rows_of(a.s_in, a.lds, r, sr);
      rows_of(a.dy, a.ldy, r, yr);
      if (LAYER) m2 = a.mean2[r];
      r2 = a.rstd2[r];
    }
    if (FAST || a.ds) rows_of(a.ds, a.ldd, r, dr);
    if (FAST || a.h) rows_of(a.h, a.ldh, r, hr);
    if (full) rows_of(a.gate, a.ldg, r, gr);
    if (post) {
      if (LAYER) m1 = a.mean1[r];
      r1 = a.rstd1[r];
    }
  };
  int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
  if (row < a.rows) load(row);
  for (; row < a.rows; row += stride) {
    float x[J][V], d[J][V], u[J][V], gate[J][V], h[J][V];
    const float mean1 = m1, rstd1 = r1, mean2 = m2, rstd2 = r2;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      Elem<T>::get(sr[j], x[j]);
      Elem<T>::get(yr[j], u[j]);
      Elem<T>::get(dr[j], d[j]);
      Elem<T>::get(hr[j], h[j]);
      Elem<T>::get(gr[j], gate[j]);
    }
    load(row + stride);
    if (pre) {
      float c[2] = {};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float g[V];
        Elem<T>::get(w2[j], g);
        second_piece<V, LAYER>(mean2, rstd2, g, left(j), x[j], u[j], dg2[j], db2[j], c);
      }
      row_means<L, LAYER>(c, width, sh);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) d[j][i] += through<LAYER>(rstd2, u[j][i], x[j][i], c);
    }
    if (FAST || a.dr)
#pragma unroll
      for (int j = 0; j < J; ++j)
        st_piece<T>(static_cast<T*>(a.dr) + row * a.lddr + col_of(j), left(j), d[j], FAST || a.nt);
    float e[2] = {};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int col = col_of(j), n = left(j);
      float g1[V], b1[V], t[V];
      Elem<T>::get(w1[j], g1);
      Elem<T>::get(o1[j], b1);
      first_piece<V, LAYER>(a, post, drop, row, col, n, mean1, rstd1, g1, b1, gate[j], h[j], d[j], t);
      if (full && a.dgate) {
        st_piece<T>(static_cast<T*>(a.dgate) + row * a.lddg + col, n, t, a.nt);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) dgt[j][i] += t[i];
      }
      if (post)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dg1[j][i] = fmaf(d[j][i], h[j][i], dg1[j][i]);
          if (LAYER) db1[j][i] += d[j][i];
          d[j][i] *= g1[i];
          e[0] = fmaf(d[j][i], h[j][i], e[0]);
          if (LAYER) e[1] += d[j][i];
        }
    }
    if (FAST || a.dh) {
      if (post) row_means<L, LAYER>(e, width, sh);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (post)
#pragma unroll
          for (int i = 0; i < V; ++i) d[j][i] = through<LAYER>(rstd1, d[j][i], h[j][i], e);
        st_piece<T>(static_cast<T*>(a.dh) + row * a.lddh + col_of(j), left(j), d[j], FAST || a.nt);
      }
    }
  }
  if (!a.part) return;
  auto sums = [&](int kind, const float(&of)[J][V]) {
    if (a.slot[kind] < 0) return;
    float* out = a.part + ((int64_t)blockIdx.x * a.slots + a.slot[kind]) * cols;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = of[j][i];
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
#pragma unroll
      for (int e = 0; e < V; e += 4)
        st_piece<float>(out + col + e, cols - col - e, reinterpret_cast<float(&)[4]>(v[e]));
    }
  };
  sums(kDg1, dg1);
  sums(kDb1, db1);
  sums(kDg2, dg2);
  sums(kDb2, db2);
  sums(kDgate, dgt);
}

// A piece of d of a row past the registers, from the means that N2 subtracts.
template <class T, bool LAYER>
__device__ __forceinline__ void wide_total(const ResArgs& a, int64_t row, int col, int n, const float (&c)[2],
                                           float (&x)[Elem<T>::V], float (&dy)[Elem<T>::V], float (&d)[Elem<T>::V]) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V;
#pragma unroll
  for (int i = 0; i < V; ++i) d[i] = 0.0f;
  if (a.ds) ld_piece<T>(static_cast<const T*>(a.ds) + row * a.ldd + col, n, d);
  if (!a.pre) return;
  float g[V], u[V], none[V], zero[V] = {}, more[2] = {};
  ld_piece<T>(static_cast<const T*>(a.s_in) + row * a.lds + col, n, x);
  ld_piece<T>(static_cast<const T*>(a.dy) + row * a.ldy + col, n, dy);
  ld_weight<T>(a.g2, col, n, 1.0f, g);
#pragma unroll
  for (int i = 0; i < V; ++i) u[i] = dy[i], none[i] = 0.0f;
  second_piece<V, LAYER>(LAYER ? a.mean2[row] : 0.0f, a.rstd2[row], g, n, x, u, none, zero, more);
#pragma unroll
  for (int i = 0; i < V; ++i) d[i] += through<LAYER>(a.rstd2[row], u[i], x[i], c);
}
template <class T, bool LAYER>
__device__ __forceinline__ void wide_first(const ResArgs& a, const Dropper& drop, int64_t row, int col, int n,
                                           float (&g1)[Elem<T>::V], float (&h)[Elem<T>::V], float (&d)[Elem<T>::V],
                                           float (&t)[Elem<T>::V]) {
  constexpr int V = Elem<T>::V;
  float b1[V], gate[V] = {};
  ld_weight<T>(a.g1, col, n, 1.0f, g1);
  ld_weight<T>(a.b1, col, n, 0.0f, b1);
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = 0.0f;
  if (a.h) ld_piece<T>(static_cast<const T*>(a.h) + row * a.ldh + col, n, h);
  if (a.gate) ld_piece<T>(static_cast<const T*>(a.gate) + row * a.ldg + col, n, gate);
  first_piece<V, LAYER>(a, a.post, drop, row, col, n, a.post && LAYER ? a.mean1[row] : 0.0f, a.post ? a.rstd1[row] : 0.0f, g1, b1,
                        gate, h, d, t);
}
template <class T, bool LAYER>
__global__ __launch_bounds__(512) void k_res_bwd_wide(ResArgs a) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V, L = 512;
  __shared__ float sh[2 * L / kWave];
  const int lane = threadIdx.x, cols = a.cols;
  const int64_t row = block_id();
  if (row >= a.rows) return;
  const Dropper drop(a.drop);
  float c[2] = {}, e[2] = {};
  if (a.pre) {
    float m = LAYER ? a.mean2[row] : 0.0f, none[V] = {}, zero[V] = {};
    for (int col = lane * V; col < cols; col += L * V) {
      float x[V], u[V], g[V];
      ld_piece<T>(static_cast<const T*>(a.s_in) + row * a.lds + col, cols - col, x);
      ld_piece<T>(static_cast<const T*>(a.dy) + row * a.ldy + col, cols - col, u);
      ld_weight<T>(a.g2, col, cols - col, 1.0f, g);
      second_piece<V, LAYER>(m, a.rstd2[row], g, cols - col, x, u, none, zero, c);
    }
    row_means<L, LAYER>(c, (float)cols, sh);
    if (a.means && lane == 0) a.means[2 * row] = c[0], a.means[2 * row + 1] = c[1];
  }
  if (!a.dr && !a.dh && !(a.dgate && a.ldg)) return;
  float x[V], dy[V], d[V], g1[V], h[V], t[V];
  if (a.post && a.dh) {
    for (int col = lane * V; col < cols; col += L * V) {
      wide_total<T, LAYER>(a, row, col, cols - col, c, x, dy, d);
      wide_first<T, LAYER>(a, drop, row, col, cols - col, g1, h, d, t);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[i] *= g1[i];
        e[0] = fmaf(d[i], h[i], e[0]);
        if (LAYER) e[1] += d[i];
      }
    }
    row_means<L, LAYER>(e, (float)cols, sh);
  }
  for (int col = lane * V; col < cols; col += L * V) {
    const int n = cols - col;
    wide_total<T, LAYER>(a, row, col, n, c, x, dy, d);
    float total[V];
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] = d[i];
    wide_first<T, LAYER>(a, drop, row, col, n, g1, h, d, t);
    // (an output may lie where an input does: all of the piece has been read)
    if (a.dr) st_piece<T>(static_cast<T*>(a.dr) + row * a.lddr + col, n, total, a.nt);
    if (a.dgate && a.ldg) st_piece<T>(static_cast<T*>(a.dgate) + row * a.lddg + col, n, t, a.nt);
    if (!a.dh) continue;
    if (a.post)
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = through<LAYER>(a.rstd1[row], d[i] * g1[i], h[i], e);
    st_piece<T>(static_cast<T*>(a.dh) + row * a.lddh + col, n, d, a.nt);
  }
}
// Their sums over rows: a thread's V columns over the rows of the block's chunk
// (blocks.x chunks, blocks.y column tiles).
template <class T, bool LAYER>
__global__ __launch_bounds__(256) void k_res_cols_wide(ResArgs a) {
#pragma clang fp contract(off)
  constexpr int V = Elem<T>::V;
  const int cols = a.cols, col = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V, n = cols - col;
  if (n <= 0) return;
  const Dropper drop(a.drop);
  float s[5][V] = {};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float c[2] = {}, x[V] = {}, dy[V] = {}, d[V], g1[V], h[V], t[V];
    if (a.pre) c[0] = a.means[2 * row], c[1] = a.means[2 * row + 1];
    wide_total<T, LAYER>(a, row, col, n, c, x, dy, d);
    wide_first<T, LAYER>(a, drop, row, col, n, g1, h, d, t);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[kDg2][i] = fmaf(dy[i], x[i], s[kDg2][i]);
      s[kDb2][i] += dy[i];
      s[kDg1][i] = fmaf(d[i], h[i], s[kDg1][i]);
      s[kDb1][i] += d[i];
      s[kDgate][i] += t[i];
    }
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    if (a.slot[k] < 0) continue;
    float* out = a.part + ((int64_t)blockIdx.x * a.slots + a.slot[k]) * cols + col;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) out[i] = s[k][i];
  }
}

// ------------------------------------------------------------ dropout
// A thread takes eight columns of a row, one call of the generator.
template <class T>
__global__ __launch_bounds__(256) void k_dropout(const T* x, int64_t ldx, const T* r, int64_t ldr, T* y, int64_t ldy,
                                                 int64_t rows, int cols, Drop d, bool nt) {
  constexpr int V = Elem<T>::V, Q = 8 / V;
  const int64_t per = (cols + 7) / 8;
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  if (row >= rows) return;
  const int col = (int)(i - row * per) * 8;
  typename Elem<T>::vec xr[Q], rr[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    xr[q] = ld_raw<T>(x + row * ldx + col + q * V, cols - col - q * V);
    if (r) rr[q] = ld_raw<T>(r + row * ldr + col + q * V, cols - col - q * V);
  }
  const Dropper drop(d);
  const unsigned keep = d.t ? drop.kept<8>(row, col) : 0xffu;
  const float grow = d.t ? d.grow : 1.0f;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
#pragma clang fp contract(off)
    float v[V], u[V];
    Elem<T>::get(xr[q], v);
    if (r) Elem<T>::get(rr[q], u);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[e] = keep >> (q * V + e) & 1 ? v[e] * grow : 0.0f;
      if (r) v[e] += u[e];
    }
    st_piece<T>(y + row * ldy + col + q * V, cols - col - q * V, v, nt);
  }
}

// ------------------------------------------------------------ column sums
// The partial sums of the wanted vectors (part [parts][slots][cols]) to their places,
// in a fixed order, as k_column_sums does for two.
struct Outs {
  void* p[5];
};
template <class T>
__global__ __launch_bounds__(512) void k_res_sums(const float* part, int parts, int slots, int cols, Outs outs) {
  __shared__ float s[32][17];
  const int c = threadIdx.x % 16, p0 = threadIdx.x / 16, n = slots * cols;
  const int col = (int)block_id() * 16 + c;
  float t[8] = {};
  if (col < n)
    for (int p = p0; p < parts; p += 256)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p + 32 * i < parts) t[i] += part[(int64_t)(p + 32 * i) * n + col];
  s[p0][c] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
  __syncthreads();
  if (p0 != 0 || col >= n) return;
  float v = 0.0f;
#pragma unroll
  for (int p = 0; p < 32; ++p) v += s[p][c];
  static_cast<T*>(outs.p[col / cols])[col % cols] = (T)v;
}

// ------------------------------------------------------------ host
// The narrowest arrangement that holds a row: lanes per row and pieces per lane; J =
// 0 past the registers.  The backward keeps up to five sums a column: twelve float32
// columns a lane fit (sixteen spilled 40 to 450 registers), sixteen of bfloat16.
template <class T, bool BWD, class F>
auto res_shape(int cols, F&& f) {
  constexpr int V = Elem<T>::V;
  const int pieces = (cols + V - 1) / V;
#define E3_SHAPE(L, J) if (pieces <= L * J) return f(std::integral_constant<int, L>{}, std::integral_constant<int, J>{})
  E3_SHAPE(8, 1);
  E3_SHAPE(16, 1);
  E3_SHAPE(32, 1);
  E3_SHAPE(64, 1);
  E3_SHAPE(64, 2);
  if constexpr (V == 4 && BWD) {
    E3_SHAPE(64, 3);
    E3_SHAPE(128, 2);
    E3_SHAPE(128, 3);
    E3_SHAPE(256, 2);
    E3_SHAPE(256, 3);
    E3_SHAPE(512, 2);
    E3_SHAPE(512, 3);
  } else if constexpr (V == 4) {
    E3_SHAPE(64, 3);
    E3_SHAPE(64, 4);
    E3_SHAPE(128, 4);
    E3_SHAPE(256, 4);
    E3_SHAPE(512, 4);
  } else {
    E3_SHAPE(128, 2);
    E3_SHAPE(256, 2);
    E3_SHAPE(512, 2);
  }
#undef E3_SHAPE
  return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 0>{});
}
// Workgroups of the backward: 512 threads per CU, each group at least one round of rows.
int res_blocks(e3_dtype t, int64_t rows, int cols) {
  auto of = [&](auto L, auto J) {
    constexpr int l = decltype(L)::value, j = decltype(J)::value, nt = kResThreads<l>, R = j > 0 ? nt / l : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(j > 0 ? 256 * 512 / nt : 256, (rows + R - 1) / R));
  };
  return t == E3_F32 ? res_shape<float, true>(cols, of) : res_shape<__bf16, true>(cols, of);
}
bool res_bwd_wide(e3_dtype t, int cols) {
  auto of = [](auto, auto J) { return decltype(J)::value == 0; };
  return t == E3_F32 ? res_shape<float, true>(cols, of) : res_shape<__bf16, true>(cols, of);
}

// Whether the spans of a backward's outputs and inputs meet.
bool inputs_written(const ResArgs& a, size_t e) {
  struct Span {
    const void* p;
    int64_t ld;
  };
  auto end = [&](const Span& s) { return reinterpret_cast<uintptr_t>(s.p) + ((a.rows - 1) * s.ld + a.cols) * e; };
  for (const Span& o : {Span{a.dr, a.lddr}, Span{a.dh, a.lddh}, Span{a.ldg ? a.dgate : nullptr, a.lddg}})
    for (const Span& i : {Span{a.ds, a.ldd}, Span{a.dy, a.ldy}, Span{a.s_in, a.lds}, Span{a.h, a.ldh}, Span{a.gate, a.ldg}})
      if (o.p && i.p && reinterpret_cast<uintptr_t>(o.p) < end(i) && reinterpret_cast<uintptr_t>(i.p) < end(o)) return true;
  return false;
}

template <class T>
e3_status res_fwd(const ResArgs& a, bool layer, hipStream_t st) {
  return res_shape<T, false>(a.cols, [&](auto L, auto J) -> e3_status {
    constexpr int l = decltype(L)::value, j = decltype(J)::value;
    if constexpr (j > 0) {
      constexpr int R = kResThreads<l> / l;
      TimedLaunch t_("residual_norm_fwd", st);
      auto* k = layer ? k_res_fwd<T, l, j, true> : k_res_fwd<T, l, j, false>;
      hipLaunchKernelGGL(k, grid_of((a.rows + R - 1) / R), dim3(kResThreads<l>), 0, st, a);
    } else {
      TimedLaunch t_("residual_norm_fwd_wide", st);
      auto* k = layer ? k_res_fwd_wide<T, true> : k_res_fwd_wide<T, false>;
      hipLaunchKernelGGL(k, grid_of(a.rows), dim3(512), 0, st, a);
    }
    E3_HIP(hipGetLastError());
    return E3_OK;
  });
}
template <class T>
e3_status res_bwd(const ResArgs& a, bool layer, hipStream_t st) {
  return res_shape<T, true>(a.cols, [&](auto L, auto J) -> e3_status {
    constexpr int l = decltype(L)::value, j = decltype(J)::value;
    if constexpr (j > 0) {
      const bool fast = a.pre && a.post && a.ds && a.h && a.dr && a.dh && !(a.gate && a.ldg) && a.nt &&
                        a.cols == l * j * Elem<T>::V;
      TimedLaunch t_(fast ? "residual_norm_bwd_stream" : "residual_norm_bwd", st);
      auto* k = fast     ? (layer ? k_res_bwd<T, l, j, true, true, true> : k_res_bwd<T, l, j, false, true, true>)
                : a.post ? (layer ? k_res_bwd<T, l, j, true, true, false> : k_res_bwd<T, l, j, false, true, false>)
                         : (layer ? k_res_bwd<T, l, j, true, false, false> : k_res_bwd<T, l, j, false, false, false>);
      hipLaunchKernelGGL(k, dim3(a.blocks), dim3(kResThreads<l>), 0, st, a);
      E3_HIP(hipGetLastError());
    } else {
      auto over_rows = [&](const ResArgs& of) {
        TimedLaunch t_("residual_norm_bwd_wide", st);
        auto* k = layer ? k_res_bwd_wide<T, true> : k_res_bwd_wide<T, false>;
        hipLaunchKernelGGL(k, grid_of(of.rows), dim3(512), 0, st, of);
      };
      // The sums read the inputs again: where outputs may lie on these, a pass for the
      // means alone (two more reads) lets the sums come first.
      const bool sums_first = a.part && inputs_written(a, sizeof(T));
      if (!sums_first) {
        over_rows(a);
      } else if (a.pre) {
        ResArgs means = a;
        means.dr = means.dh = means.dgate = nullptr;
        over_rows(means);
      }
      E3_HIP(hipGetLastError());
      if (a.part) {
        TimedLaunch t_("residual_norm_bwd_cols", st);
        const int per = 256 * Elem<T>::V;
        auto* k = layer ? k_res_cols_wide<T, true> : k_res_cols_wide<T, false>;
        hipLaunchKernelGGL(k, dim3(a.blocks, (a.cols + per - 1) / per), dim3(256), 0, st, a);
        E3_HIP(hipGetLastError());
      }
      if (sums_first) over_rows(a);
      E3_HIP(hipGetLastError());
    }
    return E3_OK;
  });
}

struct ResWs {
  size_t part, total;
};
ResWs res_ws(e3_dtype t, int64_t rows, int64_t cols) {
  ResWs w{};
  if (rows == 0) return w;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  w.part = up((size_t)res_blocks(t, rows, (int)cols) * 5 * cols * sizeof(float));
  w.total = w.part + (res_bwd_wide(t, (int)cols) ? up((size_t)rows * 2 * sizeof(float)) : 0);
  return w;
}

template <class T>
e3_status dropout(const void* x, int64_t ldx, const void* r, int64_t ldr, const Drop& d, void* y, int64_t ldy,
                  int64_t rows, int64_t cols, bool nt, const char* name, hipStream_t st) {
  TimedLaunch t_(name, st);
  hipLaunchKernelGGL(k_dropout<T>, grid_of((rows * ((cols + 7) / 8) + 255) / 256), dim3(256), 0, st,
                     static_cast<const T*>(x), ldx, static_cast<const T*>(r), ldr, static_cast<T*>(y), ldy, rows,
                     (int)cols, d, nt);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
e3_status dropout_call(e3_dtype dtype, const void* x, int64_t ldx, const void* r, int64_t ldr, double p, uint64_t seed,
                       uint64_t offset, const int64_t* counter, void* y, int64_t ldy, int64_t rows, int64_t cols,
                       const char* name, e3_stream stream) {
  if (!good_rows(dtype, rows, cols) || ldx < cols || (r && ldr < cols) || ldy < cols || !good_drop(p, counter))
    return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!good_ptr(dtype, x) || misaligned(dtype, r) || !good_ptr(dtype, y)) return E3_ERR_INVALID_ARG;
  const Drop d = drop_of(p, seed, offset, counter);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool nt = streams(dtype, rows, cols);
  return dtype == E3_F32 ? dropout<float>(x, ldx, r, ldr, d, y, ldy, rows, cols, nt, name, st)
                         : dropout<__bf16>(x, ldx, r, ldr, d, y, ldy, rows, cols, nt, name, st);
}

// The norms' weights, where a norm has none.
bool good_norms(e3_dtype t, e3_norm norm, unsigned where, const void* g1, const void* b1, const void* g2, const void* b2) {
  if ((norm != E3_NORM_RMS && norm != E3_NORM_LAYER) || where > (E3_NORM_AFTER | E3_NORM_BEFORE)) return false;
  if ((!(where & E3_NORM_AFTER) && (g1 || b1)) || (!(where & E3_NORM_BEFORE) && (g2 || b2))) return false;
  if (norm == E3_NORM_RMS && (b1 || b2)) return false;
  return !misaligned(t, g1) && !misaligned(t, b1) && !misaligned(t, g2) && !misaligned(t, b2);
}

}  // namespace

extern "C" {

e3_status e3_dropout_fwd(e3_dtype dtype, const void* x, int64_t ldx, const void* r, int64_t ldr, double p, uint64_t seed,
                         uint64_t offset, const int64_t* counter, void* y, int64_t ldy, int64_t rows, int64_t cols,
                         e3_stream stream) {
  return dropout_call(dtype, x, ldx, r, ldr, p, seed, offset, counter, y, ldy, rows, cols, "dropout_fwd", stream);
}
e3_status e3_dropout_bwd(e3_dtype dtype, const void* dy, int64_t lddy, double p, uint64_t seed, uint64_t offset,
                         const int64_t* counter, void* dx, int64_t lddx, int64_t rows, int64_t cols, e3_stream stream) {
  return dropout_call(dtype, dy, lddy, nullptr, 0, p, seed, offset, counter, dx, lddx, rows, cols, "dropout_bwd", stream);
}

e3_status e3_residual_norm_fwd(e3_dtype dtype, e3_norm norm, unsigned where, const void* h, int64_t ldh, const void* r,
                               int64_t ldr, const void* gate, int64_t ldg, float scale, double p, uint64_t seed,
                               uint64_t offset, const int64_t* counter, const void* gamma1, const void* beta1,
                               const void* gamma2, const void* beta2, float eps, void* s, int64_t lds, void* y,
                               int64_t ldy, float* mean1, float* rstd1, float* mean2, float* rstd2, int64_t rows,
                               int64_t cols, e3_stream stream) {
  const bool post = where & E3_NORM_AFTER, pre = where & E3_NORM_BEFORE;
  if (!good_rows(dtype, rows, cols) || ldh < cols || (r && ldr < cols) || (gate && ldg != 0 && ldg < cols) ||
      (s && lds < cols) || (y && ldy < cols) || !(eps >= 0.0f) || scale != scale || !good_drop(p, counter) ||
      !good_norms(dtype, norm, where, gamma1, beta1, gamma2, beta2) || (y && !pre))
    return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!good_ptr(dtype, h) || misaligned(dtype, r) || misaligned(dtype, gate) || misaligned(dtype, s) ||
      (pre && !good_ptr(dtype, y)) || (!pre && !s))
    return E3_ERR_INVALID_ARG;
  for (const float* v : {mean1, rstd1, mean2, rstd2})
    if (misaligned(E3_F32, v)) return E3_ERR_INVALID_ARG;
  ResArgs a{};
  a.h = h, a.ldh = ldh, a.res = r, a.ldr = ldr, a.gate = gate, a.ldg = ldg, a.scale = scale;
  a.drop = drop_of(p, seed, offset, counter), a.g1 = gamma1, a.b1 = beta1, a.g2 = gamma2, a.b2 = beta2, a.eps = eps;
  a.s = s, a.lds = lds, a.y = y, a.ldy = ldy, a.mean1 = mean1, a.rstd1 = rstd1, a.mean2 = mean2, a.rstd2 = rstd2;
  a.rows = rows, a.cols = (int)cols, a.post = post, a.pre = pre, a.nt = streams(dtype, rows, cols);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool layer = norm == E3_NORM_LAYER;
  return dtype == E3_F32 ? res_fwd<float>(a, layer, st) : res_fwd<__bf16>(a, layer, st);
}

e3_status e3_residual_norm_workspace_size(e3_dtype dtype, int64_t rows, int64_t cols, size_t* bwd_bytes) {
  if (!good_rows(dtype, rows, cols) || !bwd_bytes) return E3_ERR_INVALID_ARG;
  *bwd_bytes = res_ws(dtype, rows, cols).total;
  return E3_OK;
}

e3_status e3_residual_norm_bwd(e3_dtype dtype, e3_norm norm, unsigned where, const void* h, int64_t ldh, const void* s,
                               int64_t lds, const void* gate, int64_t ldg, float scale, double p, uint64_t seed,
                               uint64_t offset, const int64_t* counter, const void* gamma1, const void* beta1,
                               const void* gamma2, const float* mean1, const float* rstd1, const float* mean2,
                               const float* rstd2, const void* dy, int64_t lddy, const void* ds, int64_t ldds, void* dr,
                               int64_t lddr, void* dh, int64_t lddh, void* dgate, int64_t lddg, void* dgamma1,
                               void* dbeta1, void* dgamma2, void* dbeta2, void* ws, size_t ws_bytes, int64_t rows,
                               int64_t cols, e3_stream stream) {
  const bool post = where & E3_NORM_AFTER, pre = where & E3_NORM_BEFORE, layer = norm == E3_NORM_LAYER;
  if (!good_rows(dtype, rows, cols) || (h && ldh < cols) || (s && lds < cols) || (gate && ldg != 0 && ldg < cols) ||
      (dy && lddy < cols) || (ds && ldds < cols) || (dr && lddr < cols) || (dh && lddh < cols) ||
      (dgate && ldg != 0 && lddg < cols) || scale != scale || !good_drop(p, counter) ||
      !good_norms(dtype, norm, where, gamma1, beta1, gamma2, nullptr))
    return E3_ERR_INVALID_ARG;
  if ((dgate && !gate) || (!post && (dgamma1 || dbeta1)) || (!pre && (dgamma2 || dbeta2 || dy)) ||
      (!layer && (dbeta1 || dbeta2)))
    return E3_ERR_INVALID_ARG;
  for (const void* v : {h, s, gate, dy, ds, (const void*)dr, (const void*)dh, (const void*)dgate, (const void*)dgamma1,
                        (const void*)dbeta1, (const void*)dgamma2, (const void*)dbeta2})
    if (misaligned(dtype, v)) return E3_ERR_INVALID_ARG;
  for (const float* v : {mean1, rstd1, mean2, rstd2})
    if (misaligned(E3_F32, v)) return E3_ERR_INVALID_ARG;
  const bool later = dr || dh || dgate || dgamma1 || dbeta1;  // needs the whole of d
  if (rows > 0) {
    if (pre && (!s || !dy || !rstd2 || (layer && !mean2))) return E3_ERR_INVALID_ARG;
    if (!pre && later && !ds) return E3_ERR_INVALID_ARG;
    if (post && (dh || dgate || dgamma1 || dbeta1) && (!h || !rstd1 || (layer && !mean1))) return E3_ERR_INVALID_ARG;
    if (dgate && !h) return E3_ERR_INVALID_ARG;
  }
  ResArgs a{};
  Outs outs{};
  void* const vectors[5] = {dgamma1, dbeta1, dgamma2, dbeta2, ldg == 0 ? dgate : nullptr};
  for (int k = 0; k < 5; ++k) {
    a.slot[k] = vectors[k] ? a.slots : -1;
    if (vectors[k]) outs.p[a.slots++] = vectors[k];
  }
  const bool sums = a.slots > 0;
  const ResWs w = res_ws(dtype, rows, cols);
  if (sums && ws_bytes < w.total) return E3_ERR_WORKSPACE_TOO_SMALL;
  if (sums && w.total && (!ws || misaligned(E3_F32, ws))) return E3_ERR_INVALID_ARG;
  if (!sums && !dr && !dh && !dgate) return E3_OK;
  const bool first = dh || dgate || dgamma1 || dbeta1;  // N1's part is needed
  a.h = first && (post || dgate) ? h : nullptr, a.ldh = ldh, a.gate = first ? gate : nullptr, a.ldg = ldg, a.scale = scale;
  a.drop = first ? drop_of(p, seed, offset, counter) : Drop{}, a.g1 = gamma1, a.b1 = beta1, a.g2 = gamma2;
  a.s_in = s, a.lds = lds, a.dy = dy, a.ldy = lddy, a.ds = ds, a.ldd = ldds;
  a.mean1 = const_cast<float*>(mean1), a.rstd1 = const_cast<float*>(rstd1);
  a.mean2 = const_cast<float*>(mean2), a.rstd2 = const_cast<float*>(rstd2);
  a.dr = dr, a.lddr = lddr, a.dh = dh, a.lddh = lddh, a.dgate = dgate, a.lddg = lddg;
  a.rows = rows, a.cols = (int)cols, a.post = post && first, a.pre = pre, a.nt = streams(dtype, rows, cols);
  a.blocks = rows ? res_blocks(dtype, rows, (int)cols) : 0;
  if (sums && rows) {
    a.part = static_cast<float*>(ws);
    if (w.total > w.part) a.means = reinterpret_cast<float*>(static_cast<char*>(ws) + w.part);
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (rows) {
    const e3_status e = dtype == E3_F32 ? res_bwd<float>(a, layer, st) : res_bwd<__bf16>(a, layer, st);
    if (e != E3_OK) return e;
  }
  if (!sums) return E3_OK;
  TimedLaunch t_("residual_norm_sums", st);
  const dim3 grid = grid_of(((int64_t)a.slots * cols + 15) / 16);
  const float* part = static_cast<const float*>(ws);
  if (dtype == E3_F32)
    hipLaunchKernelGGL(k_res_sums<float>, grid, dim3(512), 0, st, part, a.blocks, a.slots, (int)cols, outs);
  else
    hipLaunchKernelGGL(k_res_sums<__bf16>, grid, dim3(512), 0, st, part, a.blocks, a.slots, (int)cols, outs);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

}  // extern "C"
