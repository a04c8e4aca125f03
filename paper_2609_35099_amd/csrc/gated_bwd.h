// Gated dense layers: the backward of narrow ones in one pass over the rows, for the
// type of the including unit.
//
//   dz = [dy u act'(g) | dy act(g)],  dx = dz W^T, dW = x^T dz, db = sum_rows dz
//
// dz never goes to memory, and in bfloat16 two terms hold 16 bits of it (one would cost
// dx and dW 1.4 to 1.7 times the error of their own rounding, and saves 4 us of 45): a
// workgroup takes blocks of 32 or 64 rows, writes their dz and x to LDS as terms
// (dense_tile.h), and its eight waves multiply both products from there, dx's with the
// terms of W in registers for good, dW's into registers that stay for all blocks; what
// is left is to add the workgroups' dW and db in order.  The next block's rows are in
// flight meanwhile.  100,003 x 64 x 128 float32 71 us and 9 for the sums, with dz
// written and two products 123; its bytes, once, at a copy's rate are 40.  bfloat16 49 in all
// of 20, 156,000 x 64 x 64 39 of 20 (float32 56 of 39).
// A round of a block is bound by its steps behind each other (loads, dz, terms to LDS,
// products, barriers): 16 waves, or two buffers of LDS with waves that form the one
// while others multiply the other, were no faster.
#pragma once
#include "gated.h"

namespace {

template <class T>
struct FusedArgs {
  const T *dy, *z, *W;
  RowsIn<T> x;
  T* dx;
  float* part;  // [workgroups][K 2 N + 2 N]: dW and db
  int64_t lddy, ldz, lddx, rows;
  int K, N, act;
  bool dw, nt;
};

template <class T>
__device__ __forceinline__ void gated_dz_piece(int act, const float (&d)[Elem<T>::V], const float (&g)[Elem<T>::V],
                                               float (&u)[Elem<T>::V], float (&e)[Elem<T>::V]) {
  constexpr int V = Elem<T>::V;
#pragma unroll
  for (int i = 0; i < V; ++i) u[i] *= d[i], e[i] = g[i];
  act_grad_piece(act, g, u);
  act_piece(act, e);
#pragma unroll
  for (int i = 0; i < V; ++i) e[i] *= d[i];
}
// One value of dz in float32 (column j of 2 N).
template <class T>
__device__ __forceinline__ float gated_dz_value(const FusedArgs<T>& a, int64_t row, int j) {
  const int n = j < a.N ? j : j - a.N;
  const float d = Elem<T>::one(a.dy[row * a.lddy + n]), g = Elem<T>::one(a.z[row * a.ldz + n]);
  return j < a.N ? d * Elem<T>::one(a.z[row * a.ldz + a.N + n]) * act_grad(a.act, g) : d * act_of(a.act, g);
}

// KB blocks of 32 columns of x, NB of each half of z; what is past K or N is zero.
template <class T, int KB, int NB, bool XQ>
struct Fused {
  static constexpr bool f32 = sizeof(T) == 4;
  static constexpr int V = Elem<T>::V, P = f32 ? 3 : 1, PZ = f32 ? 3 : 2, R = gated_fused_rows(f32, 32 * NB), RB = R / 32, NC = 64 * NB, KC = 32 * KB, WAVES = 8, THREADS = 512;
  static constexpr float kBack = f32 ? kTermBack : 1.0f;
  // pieces of a row and of a thread
  static constexpr int PR = 32 * NB / V, NP = (R * PR + THREADS - 1) / THREADS;
  static constexpr int XR = KC / V, NX = (R * XR + THREADS - 1) / THREADS;
  // dx: a wave takes one of RB KB blocks over DS of the NC / 16 reduction steps
  static constexpr int STEPS = NC / 16, UNITS = RB * KB, DS = STEPS * UNITS >= WAVES ? STEPS * UNITS / WAVES : 1;
  // dW: blocks of 32 x 32; a wave takes DB of them, or one over half of the R / 16 steps
  static constexpr int BLOCKS = KB * 2 * NB, DB = BLOCKS >= WAVES ? BLOCKS / WAVES : 1;
  static constexpr int DW_SPLIT = BLOCKS >= WAVES ? 1 : 2, DW_WAVES = BLOCKS / DB * DW_SPLIT;
  static constexpr int DW_STEPS = 2 * RB / DW_SPLIT;
  struct Shared {
    unsigned short dz[PZ][R * NC];
    unsigned short x[P][R * KC];
    float stage[WAVES][32][36];
  };
  // 16-byte slots are exchanged so that neither 16 rows at a slot nor four rows at four
  // neighbouring slots meet in a bank.
  static __device__ __forceinline__ int dz_off(int row, int slot) {
    const int x = NC >= 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
    return row * NC + (slot ^ x) * 8;
  }
  static __device__ __forceinline__ int x_off(int row, int slot) {
    return row * KC + (KC == 64 ? slot ^ (row >> 1 & 1) << 2 : slot) * 8;
  }
  // Columns c0 + l % 32 at rows k0 + 8 (l / 32) on.
  template <class Off>
  static __device__ __forceinline__ bf8v across(const unsigned short* p, Off&& off, int c0, int k0) {
    typedef __attribute__((address_space(3))) s4v* lds;
    const int l = threadIdx.x % kWave, k = k0 + 8 * (l / 32) + (l % 16) / 4, col = c0 + 16 * ((l / 16) % 2) + 4 * (l % 4);
    union {
      s4v h[2];
      bf8v f;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + off(k, col / 8) + col % 8));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + off(k + 4, col / 8) + col % 8));
    return u.f;
  }
  // The first N terms of V values, to N planes.
  template <int N>
  static __device__ __forceinline__ void put(unsigned short* p, int plane, float (&v)[V]) {
    if constexpr (f32)
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] *= kTermScale;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      unsigned b[V / 2];
#pragma unroll
      for (int k = 0; k < V / 2; ++k) b[k] = term2(v[2 * k], v[2 * k + 1]);
      if constexpr (V == 4) *reinterpret_cast<u2v*>(p + t * plane) = u2v{b[0], b[1]};
      else *reinterpret_cast<u4v*>(p + t * plane) = u4v{b[0], b[1], b[2], b[3]};
    }
  }
  // Pairs of terms, smallest products first.
  template <int PY, int PX>
  static __device__ __forceinline__ f16v products(const bf8v (&y)[PY], const bf8v (&x)[PX], f16v acc) {
#pragma unroll
    for (int s = PY + PX - 2 < 2 ? PY + PX - 2 : 2; s >= 0; --s)
#pragma unroll
      for (int p = 0; p < PX; ++p)
        if (s - p >= 0 && s - p < PY) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[s - p], x[p], acc, 0, 0, 0);
    return acc;
  }
};

// A barrier for LDS alone: __syncthreads() would wait for the loads in flight as well.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class T, int KB, int NB, bool XQ, bool FAST>
__global__ __launch_bounds__(512, 2) void k_gated_bwd(FusedArgs<T> a) {
  using F = Fused<T, KB, NB, XQ>;
  using Vec = typename Elem<T>::vec;
  constexpr int V = F::V, P = F::P;
  __shared__ __align__(16) typename F::Shared sh;
  const int tid = threadIdx.x, l = tid % kWave, w = uniform(tid / kWave), K = a.K, N = a.N;
  const int64_t blocks = (a.rows + F::R - 1) / F::R;
  // the wave's part of dx: rows rb, block kb of x's columns, reduction steps ks0 on
  const int kb = w % KB, rb = w / KB % F::RB, ks0 = w / F::UNITS * F::DS;
  bf8v wf[F::DS][P] = {};
  if (a.dx)
#pragma unroll
    for (int s = 0; s < F::DS; ++s) {
      const int j = (ks0 + s) * 16 + 8 * (l / 32), half = j / (32 * NB), n = j % (32 * NB), k = kb * 32 + l % 32;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // (loaded without a branch, so that all are in flight)
        const T u = a.W[(int64_t)imin(k, K - 1) * 2 * N + (half & 1) * N + imin(n + e, N - 1)];
        v[e] = ks0 + s < F::STEPS && k < K && n + e < N ? Elem<T>::one(u) : 0.0f;
        if (F::f32) v[e] *= kTermScale;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        u4v t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
        wf[s][p] = __builtin_bit_cast(bf8v, t);
      }
    }
  // and of dW: blocks db0 on, all steps of 16 rows or one half of them
  const int db0 = F::DW_SPLIT == 1 ? w * F::DB : w % F::BLOCKS, dstep = F::DW_SPLIT == 1 ? 0 : w / F::BLOCKS;
  f16v dw[F::DB];
#pragma unroll
  for (int j = 0; j < F::DB; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[j][e] = 0.0f;
  float sum[2][V] = {};
  // FAST: whole pieces, rows near each other; loads without a branch, so that the next
  // rows stay in flight until they are used.  Rows and columns past the end read the
  // last ones and are zeroed when they are used.
  Vec dyr[F::NP], gr[F::NP], ur[F::NP];
  typename RowsIn<T>::template Raw<XQ> xr[F::NX];
  auto load = [&](int64_t b) {
    if (b >= blocks) b = blocks - 1;
    const int64_t row0 = b * F::R;
    const int last = a.rows - row0 < F::R ? (int)(a.rows - row0) - 1 : F::R - 1;
    const T *dy = a.dy + row0 * a.lddy, *z = a.z + row0 * a.ldz;
#pragma unroll
    for (int i = 0; i < F::NP; ++i) {
      const int p = tid + i * F::THREADS, r = p / F::PR, col = p % F::PR * V;
      if constexpr (FAST) {
        const int m = imin(r, last), c = imin(col, N - V);
        dyr[i] = *reinterpret_cast<const Vec*>(dy + (unsigned)(m * (int)a.lddy + c));
        gr[i] = *reinterpret_cast<const Vec*>(z + (unsigned)(m * (int)a.ldz + c));
        ur[i] = *reinterpret_cast<const Vec*>(z + (unsigned)(m * (int)a.ldz + N + c));
      } else {
        const int n = r <= last ? N - col : 0, m = r <= last ? r : 0;
        dyr[i] = ld_raw<T>(dy + m * a.lddy + col, n);
        gr[i] = ld_raw<T>(z + m * a.ldz + col, n);
        ur[i] = ld_raw<T>(z + m * a.ldz + N + col, n);
      }
    }
    if (a.dw)
#pragma unroll
      for (int i = 0; i < F::NX; ++i) {
        const int p = tid + i * F::THREADS, r = p / F::XR, col = p % F::XR * V;
        if constexpr (FAST && !XQ) {
          xr[i] = *reinterpret_cast<const Vec*>(a.x.x + row0 * a.x.ld + (unsigned)(imin(r, last) * (int)a.x.ld + imin(col, K - V)));
        } else {
          const bool in = r <= last && col < K;
          xr[i] = a.x.template raw<XQ>(row0 + (in ? r : 0), in ? col : K, K);
        }
      }
  };
  // dz and x of the rows that were loaded (`count` of them), to LDS
  auto form = [&](int count) {
#pragma unroll
    for (int i = 0; i < F::NP; ++i) {
      const int p = tid + i * F::THREADS, r = p / F::PR, col = p % F::PR * V;
      float d[V], g[V], u[V], e[V];
      Elem<T>::get(dyr[i], d), Elem<T>::get(gr[i], g), Elem<T>::get(ur[i], u);
      gated_dz_piece<T>(a.act, d, g, u, e);
      const bool in = r < count && col < N;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        u[k] = in ? u[k] : 0.0f, e[k] = in ? e[k] : 0.0f;
        sum[0][k] += u[k], sum[1][k] += e[k];
      }
      if (r < F::R) {
        F::template put<F::PZ>(&sh.dz[0][F::dz_off(r, col / 8) + col % 8], F::R * F::NC, u);
        F::template put<F::PZ>(&sh.dz[0][F::dz_off(r, (col + 32 * NB) / 8) + col % 8], F::R * F::NC, e);
      }
    }
    if (a.dw)
#pragma unroll
      for (int i = 0; i < F::NX; ++i) {
        const int p = tid + i * F::THREADS, r = p / F::XR, col = p % F::XR * V;
        float v[V];
        RowsIn<T>::template get<XQ>(xr[i], v);
        const bool in = r < count && col < K;
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = in ? v[k] : 0.0f;
        if (r < F::R) F::template put<P>(&sh.x[0][F::x_off(r, col / 8) + col % 8], F::R * F::KC, v);
      }
  };
  // Both products of a block.  dx's sum runs over its steps in two chains, so that with
  // dW's no instruction waits for the one before it.
  auto multiply = [&]() {
    constexpr int CH = F::DS > 1 ? 2 : 1;
    f16v dx[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) dx[c][e] = 0.0f;
#pragma unroll
    for (int s = 0; s < F::DS; ++s) {
      bf8v z[F::PZ];
#pragma unroll
      for (int p = 0; p < F::PZ; ++p)
        z[p] = *reinterpret_cast<const bf8v*>(&sh.dz[p][F::dz_off(rb * 32 + l % 32, (ks0 + s) % F::STEPS * 2 + l / 32)]);
      dx[s % CH] = F::products(wf[s], z, dx[s % CH]);
    }
#pragma unroll
    for (int t = 0; t < F::DW_STEPS; ++t)
#pragma unroll
      for (int j = 0; j < F::DB; ++j) {
        const int block = db0 + j, k0 = 16 * ((dstep * F::DW_STEPS + t) % (2 * F::RB));
        bf8v x[P], z[F::PZ];
#pragma unroll
        for (int p = 0; p < P; ++p) x[p] = F::across(sh.x[p], F::x_off, block / (2 * NB) * 32, k0);
#pragma unroll
        for (int p = 0; p < F::PZ; ++p) z[p] = F::across(sh.dz[p], F::dz_off, block % (2 * NB) * 32, k0);
        dw[j] = F::products(z, x, dw[j]);
      }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f4v v{dx[0][4 * g], dx[0][4 * g + 1], dx[0][4 * g + 2], dx[0][4 * g + 3]};
      if (CH == 2) v += f4v{dx[CH - 1][4 * g], dx[CH - 1][4 * g + 1], dx[CH - 1][4 * g + 2], dx[CH - 1][4 * g + 3]};
      *reinterpret_cast<f4v*>(&sh.stage[w][l % 32][8 * g + 4 * (l / 32)]) = v * F::kBack;
    }
  };
  auto finish = [&](int64_t at) {
    if (a.dx) {
      // the waves' sums over the reduction, in order
      constexpr int SPLITS = F::STEPS / F::DS;  // (waves past them have none of it)
#pragma unroll
      for (int i = 0; i < F::NX; ++i) {
        const int p = tid + i * F::THREADS, r = p / F::XR, col = p % F::XR * V;
        const int64_t row = at * F::R + r;
        if (r >= F::R || row >= a.rows) continue;
        float v[V] = {};
#pragma unroll
        for (int q = 0; q < SPLITS; ++q)
#pragma unroll
          for (int e = 0; e < V; e += 4) {
            const f4v t = *reinterpret_cast<const f4v*>(&sh.stage[q * F::UNITS + r / 32 * KB + col / 32][r % 32][col % 32 + e]);
            v[e] += t.x, v[e + 1] += t.y, v[e + 2] += t.z, v[e + 3] += t.w;
          }
        if constexpr (F::f32) {
          float bad = 0.0f;
#pragma unroll
          for (int e = 0; e < V; ++e) bad = fmaf(v[e], 0.0f, bad);
          if (bad != 0.0f)
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (v[e] * 0.0f != 0.0f && col + e < K) {
                v[e] = 0.0f;
#pragma clang loop unroll(disable)
                for (int j = 0; j < 2 * N; ++j)
                  v[e] = fmaf(gated_dz_value(a, row, j), Elem<T>::one(a.W[(int64_t)(col + e) * 2 * N + j]), v[e]);
              }
        }
        st_piece<T>(a.dx + row * a.lddx + col, K - col, v, a.nt);
      }
    }
  };
  // A block's dx is stored after the next one's rows were used and before the loads of
  // the one after: the wait for those then finds the stores done.
  if (blockIdx.x < blocks) load(blockIdx.x);
  int64_t b = blockIdx.x;
  for (; b < blocks; b += gridDim.x) {
    form((int)(a.rows - b * F::R < F::R ? a.rows - b * F::R : F::R));
    if (b != blockIdx.x) finish(b - gridDim.x);
    load(b + gridDim.x);
    lds_barrier();
    multiply();
    lds_barrier();
  }
  if (blockIdx.x < blocks) finish(b - gridDim.x);
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * ((int64_t)K * 2 * N + 2 * N);
  if (a.dw) {
    if constexpr (F::DW_SPLIT > 1) {
      __syncthreads();
      if (dstep == 1)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f4v*>(&sh.stage[w % F::BLOCKS][l % 32][8 * g + 4 * (l / 32)]) =
              f4v{dw[0][4 * g], dw[0][4 * g + 1], dw[0][4 * g + 2], dw[0][4 * g + 3]};
      __syncthreads();
      if (dstep == 0)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f4v t = *reinterpret_cast<const f4v*>(&sh.stage[w % F::BLOCKS][l % 32][8 * g + 4 * (l / 32)]);
          dw[0][4 * g] += t.x, dw[0][4 * g + 1] += t.y, dw[0][4 * g + 2] += t.z, dw[0][4 * g + 3] += t.w;
        }
    }
    __syncthreads();
    // by way of the wave's staging, so that rows are written in runs of 128 bytes
    if (dstep == 0)
#pragma unroll
      for (int j = 0; j < F::DB; ++j) {
        const int block = db0 + j, nb = block % (2 * NB), half = nb / NB;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f4v*>(&sh.stage[w][l % 32][8 * g + 4 * (l / 32)]) =
              f4v{dw[j][4 * g], dw[j][4 * g + 1], dw[j][4 * g + 2], dw[j][4 * g + 3]} * F::kBack;
        Rows32<float, 1>::wait();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * i + l / 8, k = block / (2 * NB) * 32 + r, n = nb % NB * 32 + 4 * (l % 8);
          const f4v s = *reinterpret_cast<const f4v*>(&sh.stage[w][r][4 * (l % 8)]);
          float v[4] = {s.x, s.y, s.z, s.w};
          if constexpr (F::f32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v[e] * 0.0f != 0.0f && k < K && n + e < N) {
                v[e] = 0.0f;
#pragma clang loop unroll(disable)
                for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x)
#pragma clang loop unroll(disable)
                  for (int64_t row = b * F::R; row < (b + 1) * F::R && row < a.rows; ++row)
                    v[e] = fmaf(a.x.value(row, k, K), gated_dz_value(a, row, half * N + n + e), v[e]);
              }
          }
          if (k < K) st_piece<float>(part + (int64_t)k * 2 * N + half * N + n, N - n, v);
        }
        Rows32<float, 1>::wait();
      }
  }
  // db: the threads of a piece, in order
  constexpr int GROUPS = F::THREADS < F::R * F::PR ? F::THREADS / F::PR : F::R;
  static_assert(GROUPS * F::NC * sizeof(float) <= sizeof(sh.stage));
  float* fold = &sh.stage[0][0][0];
  __syncthreads();
  if (tid / F::PR < GROUPS)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < V; ++k) fold[tid / F::PR * F::NC + h * 32 * NB + tid % F::PR * V + k] = sum[h][k];
  __syncthreads();
  for (int c = tid; c < F::NC; c += F::THREADS) {
    const int half = c / (32 * NB), n = c % (32 * NB);
    if (n >= N) continue;
    float v = 0.0f;
    for (int q = 0; q < GROUPS; ++q) v += fold[q * F::NC + c];
    part[(int64_t)K * 2 * N + half * N + n] = v;
  }
}

template <class T, int KB, int NB>
e3_status gated_bwd_fused_of(const FusedArgs<T>& a, int groups, hipStream_t st) {
  TimedLaunch t_("gated_bwd_fused", st);
  constexpr int V = Elem<T>::V;
  constexpr int64_t near = 1 << 25;  // strides whose 64 rows and two halves of z stay in 31 bits
  const bool packed = a.dw && !a.x.x;
  const bool fast = a.N % V == 0 && a.lddy < near && a.ldz < near && (!a.dw || packed || (a.K % V == 0 && a.x.ld < near));
  auto* k = packed ? (fast ? k_gated_bwd<T, KB, NB, true, true> : k_gated_bwd<T, KB, NB, true, false>)
                   : (fast ? k_gated_bwd<T, KB, NB, false, true> : k_gated_bwd<T, KB, NB, false, false>);
  hipLaunchKernelGGL(k, dim3((unsigned)groups), dim3(512), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
template <class T>
e3_status gated_bwd_fused(const GatedCall& c) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  const int groups = gated_fused_groups(t, c.M, c.N);
  FusedArgs<T> a{};
  a.dy = static_cast<const T*>(c.dy), a.z = static_cast<const T*>(c.z_in), a.W = static_cast<const T*>(c.W);
  a.x = {static_cast<const T*>(c.x), c.ldx, c.xq, c.xc}, a.dx = static_cast<T*>(c.dx), a.lddy = c.lddy, a.ldz = c.ldz;
  a.lddx = c.lddx, a.rows = c.M, a.K = (int)c.K, a.N = (int)c.N, a.act = c.act, a.dw = c.dW != nullptr;
  a.nt = streams(t, c.M, c.K);
  if (c.dW || c.db) a.part = reinterpret_cast<float*>(c.ws);
  auto with = [&](auto KB) {
    constexpr int kb = decltype(KB)::value;
    return c.N <= 32   ? gated_bwd_fused_of<T, kb, 1>(a, groups, c.st)
           : c.N <= 64 ? gated_bwd_fused_of<T, kb, 2>(a, groups, c.st)
                       : gated_bwd_fused_of<T, kb, 4>(a, groups, c.st);
  };
  const e3_status s = c.K <= 32 ? with(std::integral_constant<int, 1>{}) : with(std::integral_constant<int, 2>{});
  if (s != E3_OK || !a.part) return s;
  const int64_t kn = c.K * 2 * c.N;
  return column_sums(t, a.part, groups, kn + 2 * c.N, kn, kn + 2 * c.N, c.dW, c.db, c.st);
}

}  // namespace
