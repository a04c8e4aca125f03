// Gated dense layers, for the type of the including unit.
//
//   [g | u] = x W + b,  y = act(g) u           W [K, 2 N]
//   dz = [dy u act'(g) | dy act(g)],  dx = dz W^T, dW = x^T dz, db = sum_rows dz
//
// Forward: a tile takes the columns of both halves in turns of 32 (kPaired), so
// that the two of a pair meet in one wave's staging and neither g nor u goes to
// memory unless it is kept.  Backward: narrow layers form dz block by block in LDS, in
// one pass over the rows (gated_bwd.h); otherwise it is written once, by the pass that sums
// db, and the products are those of a dense layer of 2 N columns.
#pragma once
#include "dense.h"

// A gated call, checked.
struct GatedCall {
  e3_dtype dtype;
  const void *x, *W, *bias;
  int64_t ldx;
  int act;
  void *y, *z;
  int64_t ldy, ldz;
  int8_t *gq, *uq, *yq;
  uint8_t *gc, *uc, *yc;
  // backward
  const void *dy, *z_in;
  const int8_t *xq, *gq_in, *uq_in;
  const uint8_t *xc, *gc_in, *uc_in;
  void *dx, *dW, *db;
  int64_t lddy, lddx;
  char* ws;
  int64_t M, K, N;
  hipStream_t st;
};
e3_status gated_fwd_f32(const GatedCall& c);
e3_status gated_fwd_bf16(const GatedCall& c);
e3_status gated_bwd_fused_f32(const GatedCall& c);
e3_status gated_bwd_fused_bf16(const GatedCall& c);

namespace {

struct GatedArgs {
  Side a, b;  // x [rows, red], W [red, 2 cols]
  int64_t rows, red;
  int cols;   // of y
  const void* bias;
  int act;
  void *y, *z;
  int64_t ldy, ldz;
  int8_t *gq, *uq, *yq;
  uint8_t *gc, *uc, *yc;
  int64_t chunks;  // row chunks of the panel
  float* part;     // partial sums of z, [splits][rows][2 cols], instead of the epilogue
  int red_chunk;   // reduction indexes of a split
  bool nt;
};

// What follows the sums of a piece of a row: columns col on of y.  The lanes of a
// group of 32 columns take part together, also where rows (ok) or columns end.
template <class T>
struct GatedTail {
  static constexpr int V = Elem<T>::V;
  float bg[V], bu[V];
  __device__ __forceinline__ GatedTail(const GatedArgs& a, int col) {
#pragma unroll
    for (int i = 0; i < V; ++i) bg[i] = bu[i] = 0.0f;
    if (!a.bias) return;
    ld_piece<T>(static_cast<const T*>(a.bias) + col, a.cols - col, bg);
    ld_piece<T>(static_cast<const T*>(a.bias) + a.cols + col, a.cols - col, bu);
  }
  // FAST: the piece is inside the row, y is the only output (plain()).
  template <bool FAST = false, bool NT = true>
  __device__ __forceinline__ void out(const GatedArgs& a, int64_t row, bool ok, int col, float (&g)[V],
                                      float (&u)[V]) const {
    const int n = FAST ? V : ok ? a.cols - col : 0;
    const int64_t groups = (a.cols + kGroup - 1) / kGroup;
    auto pack = [&](const float(&v)[V], int8_t* q, uint8_t* c) {
      pack8_piece<V>(v, col, n, q + row * a.cols, c + row * groups);
    };
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] += bg[i], u[i] += bu[i];
    if (!FAST && a.z) {
      T* z = static_cast<T*>(a.z) + row * a.ldz + col;
      st_piece<T>(z, n, g, a.nt);
      st_piece<T>(z + a.cols, n, u, a.nt);
    }
    if (!FAST && a.gq) pack(g, a.gq, a.gc), pack(u, a.uq, a.uc);
    act_piece(a.act, g);
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = Elem<T>::round(g[i] * u[i]);
    T* y = static_cast<T*>(a.y) + row * a.ldy + col;
    if constexpr (FAST && NT) __builtin_nontemporal_store(Elem<T>::put(g), reinterpret_cast<typename Elem<T>::vec*>(y));
    else if constexpr (FAST) *reinterpret_cast<typename Elem<T>::vec*>(y) = Elem<T>::put(g);
    else st_piece<T>(y, n, g, a.nt);
    if (!FAST && a.yq) pack(g, a.yq, a.yc);
  }
  static bool plain(const GatedArgs& a) { return !a.z && !a.gq && !a.yq; }
};

// A sum again from memory, in float32 (half 0: g, 1: u).
template <class T>
__device__ __forceinline__ float gated_again(const GatedArgs& a, int64_t row, int col, int half) {
  float sum = 0.0f;
  const T* x = static_cast<const T*>(a.a.p) + row * a.a.ld;
  const T* w = static_cast<const T*>(a.b.p) + (int64_t)half * a.cols + col;
#pragma clang loop unroll(disable)
  for (int64_t k = 0; k < a.red; ++k) sum = fmaf(Elem<T>::one(x[k]), Elem<T>::one(w[k * a.b.ld]), sum);
  return sum;
}

// The lane's first column among 16 RN of y.
template <class T, int RN>
__device__ __forceinline__ int gated_col() {
  constexpr int V = Elem<T>::V;
  return threadIdx.x % kWave % (16 * RN / V) * V;
}
// The results of rows row0 to row0 + 31 and 16 RN columns of y from col0 on: blocks
// of 32 columns of g and of u in turn.
template <class T, int RN, bool FAST = false, bool NT = true>
__device__ __forceinline__ void gated_rows32(const GatedArgs& a, const GatedTail<T>& tail, int64_t row0, int col0,
                                             float (*out)[32 * RN + 4], const f16v (&acc)[RN]) {
  using R = Rows32<T, RN>;
  constexpr int V = R::V, PER = 16 * RN / V, PASS = kWave / PER, N = 32 / PASS;
  const int l = threadIdx.x % kWave, oc = gated_col<T, RN>(), lr = l / PER, at = oc / 32 * 64 + oc % 32;
  R::put(out, acc);
  if constexpr (sizeof(T) == 4) {
    if (R::bad(acc))
      R::mend(out, [&](int r, int c) {
        const int col = col0 + c / 64 * 32 + c % 32;
        return row0 + r < a.rows && col < a.cols ? gated_again<T>(a, row0 + r, col, c / 32 % 2) : 0.0f;
      });
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = i * PASS + lr;
    float g[V], u[V];
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      *reinterpret_cast<f4v*>(&g[e]) = *reinterpret_cast<const f4v*>(&out[r][at + e]);
      *reinterpret_cast<f4v*>(&u[e]) = *reinterpret_cast<const f4v*>(&out[r][at + 32 + e]);
    }
    tail.template out<FAST, NT>(a, row0 + r, FAST || row0 + r < a.rows, col0 + oc, g, u);
  }
  __builtin_amdgcn_wave_barrier();
}
template <class T, int RN, bool FAST = false, bool NT = true>
__device__ __forceinline__ void gated_rows32(const GatedArgs& a, int64_t row0, int col0, float (*out)[32 * RN + 4],
                                             const f16v (&acc)[RN]) {
  const GatedTail<T> tail(a, col0 + gated_col<T, RN>());
  gated_rows32<T, RN, FAST, NT>(a, tail, row0, col0, out, acc);
}

// Tiles by type and size, as TileOf's; every wave has 64 columns of z, 32 of y.  bfloat16
// 128 x 128 in steps of 32, so that three workgroups fit a CU: 5,003 x 515 x 1,021 30
// us against 34 with two and steps of 64, 10,007 rows 49 against 53.
template <class T, int B>
struct GatedTileOf {
  static constexpr bool f32 = sizeof(T) == 4;
  static constexpr int BM = f32 && B == 128 ? 64 : B, BN = B == 256 ? 128 : B;
  static constexpr int WM = B == 256 ? 4 : 2, WN = BN / 64;
  static constexpr int BK = f32 || B >= 128 ? 32 : 64, THREADS = WM * WN * kWave, OCC = B == 256 ? 4 : f32 ? 2 : 3;
  using type = Tile<T, kAlong, kPaired, BM, BN, BK, WM, WN, kFull, kFull, false, f32 ? 1 : 2>;
};
template <class T, int B>
__global__ __launch_bounds__((GatedTileOf<T, B>::THREADS), (GatedTileOf<T, B>::OCC)) void k_gated(GatedArgs a) {
  using O = GatedTileOf<T, B>;
  using Tl = typename O::type;
  __shared__ __align__(16) typename Tl::Shared sh;
  const int64_t tm = (a.rows + O::BM - 1) / O::BM, u = block_id();
  const int tn = (a.cols + O::BN / 2 - 1) / (O::BN / 2);
  if (u >= tm * tn) return;
  const TileAt at = tile_at(u, tm, tn);
  const int64_t r0 = at.m * O::BM;
  const int c0 = at.n * (O::BN / 2);
  Tl t;
  t.template run<false>(sh, {a.a, a.b, {}, 0}, r0, a.rows, c0, a.cols, 0, a.red);
  t.finish(sh, [&](int r, int c, auto out, auto& acc) { gated_rows32<T, Tl::RN>(a, r0 + r, c0 + c / 2, out, acc); });
}

// bfloat16 with operands straight to LDS.  (A template, so that only its unit compiles it.)
template <class T>
__global__ __launch_bounds__(512, 2) void k_gated_direct(GatedArgs a) {
  static_assert(sizeof(T) == 2);
  using Tl = DirectTile<kAlong, kPaired>;
  __shared__ __align__(16) Tl::Buf s0, s1;
  const int64_t tm = (a.rows + Tl::BM - 1) / Tl::BM, u = block_id();
  const int tn = (a.cols + Tl::BN / 2 - 1) / (Tl::BN / 2);
  if (u >= tm * tn) return;
  const TileAt at = tile_at(u, tm, tn);
  const int64_t r0 = at.m * Tl::BM;
  const int c0 = at.n * (Tl::BN / 2);
  // (loaded here, so that no wait for a load is one for stores)
  const GatedTail<T> tail(a, c0 + Tl::col0() / 2 + gated_col<T, Tl::RN>());
  Tl t;
  t.run(s0, s1, a.a, a.b, r0, a.rows, c0, a.cols, 0, a.red);
  auto* out = Tl::stage(s0, s1);
  each_of([&](auto i) {
    gated_rows32<T, Tl::RN>(a, tail, r0 + Tl::row0() + 32 * i, c0 + Tl::col0() / 2, out, t.acc[i]);
  }, std::make_integer_sequence<int, Tl::RM>{});
}

// Short reductions over many rows, as k_dense_panel: a wave keeps the terms of 32
// columns of g and of u and walks row blocks.
template <class T, int KK, bool FAST, bool NT>
__global__ __launch_bounds__(256, 2) void k_gated_panel(GatedArgs a) {
  using R = Rows32<T, 2>;
  constexpr bool f32 = sizeof(T) == 4;
  constexpr int V = Elem<T>::V, P = f32 ? 3 : 1, Q = 8 / V;
  __shared__ __align__(16) float out[4][32][R::PITCH];
  const int l = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), K = (int)a.red;
  const int groups = (a.cols + 31) / 32;
  const int64_t w = block_id() * 4 + wave, chunk = w / groups;
  if (chunk >= a.chunks) return;
  const int col0 = (int)(w % groups) * 32;
  const int h = 8 * (l / 32);
  bf8v wf[P][KK][2];
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = col0 + l % 32;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // (loaded without a branch, so that all are in flight: 64 waits took 20 us)
        const int at = 16 * k + h + e;
        const T u = static_cast<const T*>(a.b.p)[imin(at, K - 1) * a.b.ld + c * a.cols + imin(col, a.cols - 1)];
        v[e] = at < K && col < a.cols ? Elem<T>::one(u) : 0.0f;
        if (f32) v[e] *= kTermScale;
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        u4v t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
        wf[p][k][c] = __builtin_bit_cast(bf8v, t);
      }
    }
  typename Elem<T>::vec x[KK][Q];
  const T* xp = static_cast<const T*>(a.a.p);
  auto load = [&](auto fast, int64_t block) {
    constexpr bool F = decltype(fast)::value;
    const int last = F ? 31 : a.rows - block * 32 < 32 ? (int)(a.rows - block * 32) - 1 : 31;
    const int64_t m = imin(l % 32, last);
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int at = 16 * k + h + q * V;
        x[k][q] = ld_raw<T>(xp + block * 32 * a.a.ld + (m * a.a.ld + at), F ? V : K - at);
      }
  };
  bf8v xf[P][KK];
  auto terms = [&]() {
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      if constexpr (!f32) {
        xf[0][k] = __builtin_bit_cast(bf8v, x[k][0]);
      } else {
        float v[8];
#pragma unroll
        for (int q = 0; q < Q; ++q) Elem<T>::get(x[k][q], reinterpret_cast<float(&)[V]>(v[q * V]));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= kTermScale;
#pragma unroll
        for (int p = 0; p < P; ++p) {
          u4v t;
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
          xf[p][k] = __builtin_bit_cast(bf8v, t);
        }
      }
    }
  };
  auto product = [&](auto fast, int64_t block) {
    f16v acc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[c][e] = 0.0f;
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int s = 2 * P - 2 < 2 ? 2 * P - 2 : 2; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const int q = s - p;
          if (q < 0 || q >= P) continue;
#pragma unroll
          for (int c = 0; c < 2; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[q][k][c], xf[p][k], acc[c], 0, 0, 0);
        }
    gated_rows32<T, 2, decltype(fast)::value, NT>(a, block * 32, col0, out[wave], acc);
  };
  // FAST: whole row blocks by a loop without branches around loads and stores, and
  // what is left of the rows after it
  const int64_t blocks = FAST ? a.rows / 32 : (a.rows + 31) / 32;
  const std::integral_constant<bool, FAST> fast;
  if (chunk < blocks) {
    // a round ends with loads and begins with stores, so that its wait for the
    // loads of the one before leaves its own stores in flight; blocks past the
    // end load the last one again
    auto at = [&](int64_t b) { return b < blocks ? b : blocks - 1; };
    load(fast, chunk);
    terms();
    load(fast, at(chunk + a.chunks));
    for (int64_t block = chunk; block < blocks; block += a.chunks) {
      product(fast, block);
      terms();
      load(fast, at(block + 2 * a.chunks));
    }
  }
  if (FAST && a.rows % 32 && chunk == blocks % a.chunks) {
    load(std::false_type{}, blocks);
    terms();
    product(std::false_type{}, blocks);
  }
}

// The same in float32 for whole pieces and y alone: the terms of W lie in LDS for the
// workgroup's waves, and each forms a row block's terms, a third of the vector work,
// once for NG groups of 32 columns of y instead of once for each.  Against the kernel
// above, us: 156,000 x 64 x 64 24 and 30, 624,000 70 and 92, 1,248,000 x 32 x 128 194 and
// 223; bfloat16, which has no terms to form, 17 and 14, 42 and 37 (float32 alone has it).
// A CU holds one workgroup, by its 116 KB of LDS: two waves a SIMD, whose loads, terms,
// products and stores follow each other.  Of a SIMD's busy cycles at 156,000 x 64 x 64 vector
// instructions take 49% (920 for 32 rows, 280 of them for the terms of x, most of the others
// for the epilogue) and matrix instructions 38%.
template <int KK, int NG, bool NT>
__global__ __launch_bounds__(512, 2) void k_gated_walk(GatedArgs a) {
  using R = Rows32<float, 2>;
  constexpr int V = Elem<float>::V, P = 3, Q = 8 / V, WAVES = 8;
  __shared__ __align__(16) bf8v wf[NG][KK][2][P][kWave];
  __shared__ __align__(16) float out[WAVES][32][R::PITCH];
  const int l = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave), h = 8 * (l / 32);
  const int col0 = (int)blockIdx.y * 32 * NG;
  for (int f = wave; f < NG * KK * 2; f += WAVES) {
    const int c = f % 2, k = f / 2 % KK, g = f / 2 / KK;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = static_cast<const float*>(a.b.p)[(16 * k + h + e) * a.b.ld + c * a.cols + col0 + 32 * g + l % 32] * kTermScale;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      u4v t;
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
      wf[g][k][c][p][l] = __builtin_bit_cast(bf8v, t);
    }
  }
  __syncthreads();
  Elem<float>::vec x[KK][Q];
  const float* xp = static_cast<const float*>(a.a.p);
  auto load = [&](auto fast, int64_t block) {
    constexpr bool F = decltype(fast)::value;
    const int last = F ? 31 : (int)(a.rows - block * 32) - 1;
    const int64_t m = imin(l % 32, last);
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int q = 0; q < Q; ++q) x[k][q] = ld_raw<float>(xp + block * 32 * a.a.ld + (m * a.a.ld + 16 * k + h + q * V), V);
  };
  bf8v xf[P][KK];
  auto terms = [&]() {
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      float v[8];
#pragma unroll
      for (int q = 0; q < Q; ++q) Elem<float>::get(x[k][q], reinterpret_cast<float(&)[V]>(v[q * V]));
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= kTermScale;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        u4v t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = term2(v[2 * e], v[2 * e + 1]);
        xf[p][k] = __builtin_bit_cast(bf8v, t);
      }
    }
  };
  auto product = [&](auto fast, int64_t block) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      f16v acc[2];
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[c][e] = 0.0f;
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        bf8v y[2][P];
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int p = 0; p < P; ++p) y[c][p] = wf[g][k][c][p][l];
#pragma unroll
        for (int s = 2; s >= 0; --s)
#pragma unroll
          for (int p = 0; p < P; ++p) {
            const int q = s - p;
            if (q < 0 || q >= P) continue;
#pragma unroll
            for (int c = 0; c < 2; ++c) acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[c][q], xf[p][k], acc[c], 0, 0, 0);
          }
      }
      gated_rows32<float, 2, decltype(fast)::value, NT>(a, block * 32, col0 + 32 * g, out[wave], acc);
    }
  };
  const int64_t blocks = a.rows / 32, stride = (int64_t)gridDim.x * WAVES;
  const std::true_type fast;
  const int64_t first = (int64_t)blockIdx.x * WAVES + wave;
  if (first < blocks) {
    // rounds as k_gated_panel's
    auto at = [&](int64_t b) { return b < blocks ? b : blocks - 1; };
    load(fast, first);
    terms();
    load(fast, at(first + stride));
    for (int64_t block = first; block < blocks; block += stride) {
      product(fast, block);
      terms();
      load(fast, at(block + 2 * stride));
    }
  }
  if (a.rows % 32 && first == blocks % stride) {
    load(std::false_type{}, blocks);
    terms();
    product(std::false_type{}, blocks);
  }
}

// At most MR <= 8 rows, as k_dense_few: W is read once, straight to registers, and
// that is what bounds it.  A workgroup takes 32 columns of y.
template <class T, int MR>
__global__ __launch_bounds__(512) void k_gated_few(GatedArgs a) {
  constexpr int V = Elem<T>::V, C = 32 / V, G = 512 / C, WAVES = 512 / kWave;
  __shared__ float s[WAVES][2][MR][32];
  const int cl = threadIdx.x % C, g = threadIdx.x / C, col = (int)blockIdx.x * 32 + cl * V, n = a.cols - col;
  const int kbegin = (int)blockIdx.y * a.red_chunk, K = imin(kbegin + a.red_chunk, (int)a.red);
  const T* W = static_cast<const T*>(a.b.p);
  const T* x = static_cast<const T*>(a.a.p);
  float v[2][MR][V] = {};
  constexpr int U = MR > 4 ? 4 : 8;       // reduction indexes in flight
  // several rows of x by way of LDS (loaded value by value beside W, eight took a third of
  // the time: 1,024 to 4,096 bfloat16 21 us against 29; one row is faster without, 10.5, 11.5)
  constexpr bool STAGE = MR > 1;
  constexpr int KX = STAGE ? 8192 / MR : 1 << 30;
  __shared__ float xs[MR][STAGE ? KX : 1];
  for (int kc = kbegin; kc < K; kc = STAGE ? kc + KX : K) {
    const int ke = STAGE ? imin(kc + KX, K) : K;
    if constexpr (STAGE) {
      if (kc != kbegin) __syncthreads();
#pragma unroll
      for (int m = 0; m < MR; ++m)
        for (int k = threadIdx.x; k < ke - kc; k += 512) xs[m][k] = m < a.rows ? Elem<T>::one(x[m * a.a.ld + kc + k]) : 0.0f;
      __syncthreads();
    }
    for (int k0 = kc + g; k0 < ke; k0 += G * U) {
      typename Elem<T>::vec w[U][2];
      T own[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int k = k0 + j * G;
        if (k < ke) {
          if (!STAGE) own[j] = x[k];
          w[j][0] = ld_raw<T>(W + k * a.b.ld + col, n);
          w[j][1] = ld_raw<T>(W + k * a.b.ld + a.cols + col, n);
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (k0 + j * G < ke) {
          float u[MR];
#pragma unroll
          for (int m = 0; m < MR; ++m) u[m] = STAGE ? xs[m][k0 + j * G - kc] : Elem<T>::one(own[j]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float t[V];
            Elem<T>::get(w[j][h], t);
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
              for (int i = 0; i < V; ++i) v[h][m][i] = fmaf(u[m], t[i], v[h][m][i]);
          }
        }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float t = sum_strided<C>(v[h][m][i]);
        if (threadIdx.x % kWave < C) s[threadIdx.x / kWave][h][m][cl * V + i] = t;
      }
  __syncthreads();
  if (threadIdx.x >= MR * C) return;
  float t[2][V] = {};
  for (int q = 0; q < WAVES; ++q)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < V; ++i) t[h][i] += s[q][h][g][cl * V + i];
  if (a.part) {
    if (g >= a.rows) return;
    float* p = a.part + ((int64_t)blockIdx.y * a.rows + g) * 2 * a.cols + col;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < V; e += 4)
        st_piece<float>(p + (int64_t)h * a.cols + e, n - e, reinterpret_cast<float(&)[4]>(t[h][e]));
    return;
  }
  GatedTail<T>(a, col).out(a, g, g < a.rows, col, t[0], t[1]);
}

// Partial sums of z from the splits of its reduction, in order, and the epilogue.
template <class T>
__global__ __launch_bounds__(256) void k_gated_join(GatedArgs a, const float* part, int splits) {
  constexpr int V = Elem<T>::V;
  const int per = (a.cols + kGroup - 1) / kGroup * (kGroup / V);
  const int64_t i = block_id() * 256 + threadIdx.x, row = div_small(i, per);
  const int col = (int)(i - row * per) * V;
  const int n = row < a.rows ? a.cols - col : 0;
  const int64_t pitch = a.rows * 2 * a.cols;
  float v[2][V] = {};
  const float* p = part + (row * 2 * a.cols + col);
  for (int s = 0; s < splits; s += 4) {
    float u[4][2][V];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < V; e += 4)
          ld_piece<float>(p + (s + j) * pitch + (int64_t)h * a.cols + e, s + j < splits ? n - e : 0,
                          reinterpret_cast<float(&)[4]>(u[j][h][e]));
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < V; ++e) v[h][e] += u[j][h][e];
  }
  GatedTail<T>(a, col).out(a, row, row < a.rows, col, v[0], v[1]);
}

// ------------------------------------------------------------ host
constexpr int kGatedThin = 16, kGatedFew = 8;
// How a forward goes.
enum class GatedWay { few, panel, split, tile };
GatedWay gated_way(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  if (M <= kGatedFew) return GatedWay::few;
  // (a reduction this short has no whole piece to read in the tile's way)
  const bool p = t == E3_F32 ? panel<float>(M, 2 * N, K) : panel<__bf16>(M, 2 * N, K);
  if (p || K <= kGatedThin) return GatedWay::panel;
  return dense_cut(t, M, 2 * N, K, kForward).splits > 1 ? GatedWay::split : GatedWay::tile;
}
// Splits of a long reduction where a few rows' columns leave most of the card idle (one
// row of 4,096 to 1,024 bfloat16 13 us with eight, join included, 32 without; 1,024 to
// 1,024 float32 7 either way).
int gated_few_splits(int64_t K, int64_t N) {
  const int64_t tiles = (N + 31) / 32;
  return tiles > 64 || K < 2048 ? 1 : (int)std::min<int64_t>({256 / tiles, K / 256, 32});
}
size_t gated_fwd_ws(e3_dtype t, int64_t M, int64_t K, int64_t N) {
  if (M == 0) return 0;
  if (M <= kGatedFew) {
    const int s = gated_few_splits(K, N);
    return s > 1 ? up256((size_t)s * M * 2 * N * sizeof(float)) : 0;
  }
  if (gated_way(t, M, K, N) != GatedWay::split) return 0;
  return cut_bytes(dense_cut(t, M, 2 * N, K, kForward), M, 2 * N);
}

// Backward in one pass over the rows (gated_bwd.h): layers whose dW fits the registers of
// a workgroup, from z in full.  (dy and x hold a piece at least.)
bool gated_fused(int64_t M, int64_t K, int64_t N) { return K <= 64 && N <= 128 && M * K >= 8 && M * N >= 8; }
// Rows of its blocks: such that the workgroup's threads have a piece each (156,000 x 64 x
// 64 bfloat16 40 us with 64 rows, 48 with 32; 100,003 rows 32 and 35).
constexpr int gated_fused_rows(bool f32, int64_t N) { return N <= (f32 ? 32 : 64) ? 64 : 32; }
// Its workgroups: one per CU.
int gated_fused_groups(e3_dtype t, int64_t M, int64_t N) {
  const int rows = gated_fused_rows(t == E3_F32, N);
  return (int)std::min<int64_t>((M + rows - 1) / rows, 256);
}

// Whether k_gated_walk takes it: whole steps and groups of columns, and y alone.  (With z,
// as a training step has it, k_gated_panel runs with branches around its stores: 156,000 x
// 64 x 64 float32 38 us, its bytes at a copy's rate 31, bfloat16 19 and 16; 624,000 127 and
// 125, 65 and 63.)
bool gated_walks(const GatedArgs& a) {
  return a.rows >= 32 && GatedTail<float>::plain(a) && (a.red == 32 || a.red == 64) && a.cols % 64 == 0;
}
template <int KK, int NG>
e3_status gated_walk(const GatedArgs& a, hipStream_t st) {
  TimedLaunch t_("gated_fwd_walk", st);
  const unsigned tiles = (unsigned)(a.cols / (32 * NG));  // of columns; a workgroup per CU among them
  const int64_t rows = std::min<int64_t>((a.rows + 255) / 256, std::max<int64_t>(1, 256 / tiles));
  auto* k = a.nt ? k_gated_walk<KK, NG, true> : k_gated_walk<KK, NG, false>;
  hipLaunchKernelGGL(k, dim3((unsigned)rows, tiles), dim3(512), 0, st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

template <class T>
e3_status gated_panel(GatedArgs a, hipStream_t st) {
  if constexpr (sizeof(T) == 4) {
    if (gated_walks(a))
      return a.red == 64 ? gated_walk<4, 2>(a, st) : a.cols % 128 == 0 ? gated_walk<2, 4>(a, st) : gated_walk<2, 2>(a, st);
  }
  // two workgroups per CU, each wave on row blocks of its own
  const int64_t groups = (a.cols + 31) / 32;
  a.chunks = std::min<int64_t>((a.rows + 31) / 32, std::max<int64_t>(1, 2048 / groups));
  const int64_t blocks = (a.chunks * groups + 3) / 4;
  TimedLaunch t_("gated_fwd_panel", st);
  auto go = [&](auto KK) {
    constexpr int kk = decltype(KK)::value;
    const bool fast = a.red == 16 * kk && a.cols % 32 == 0 && GatedTail<T>::plain(a);
    auto* k = !fast ? k_gated_panel<T, kk, false, false> : a.nt ? k_gated_panel<T, kk, true, true> : k_gated_panel<T, kk, true, false>;
    hipLaunchKernelGGL(k, grid_of(blocks), dim3(256), 0, st, a);
  };
  if (a.red <= 16) go(std::integral_constant<int, 1>{});
  else if (a.red <= 32) go(std::integral_constant<int, 2>{});
  else if (sizeof(T) == 4 && a.red <= 48) go(std::integral_constant<int, 3>{});
  else if (a.red <= 64) go(std::integral_constant<int, 4>{});
  else if constexpr (sizeof(T) == 2) {
    if (a.red <= 96) go(std::integral_constant<int, 6>{});
    else go(std::integral_constant<int, 8>{});
  }
  E3_HIP(hipGetLastError());
  return E3_OK;
}

template <class T>
e3_status gated_join(const GatedArgs& a, const float* part, int splits, hipStream_t st) {
  TimedLaunch t_("gated_fwd_join", st);
  const int64_t per = (a.cols + kGroup - 1) / kGroup * (kGroup / Elem<T>::V);
  hipLaunchKernelGGL(k_gated_join<T>, grid_of((a.rows * per + 255) / 256), dim3(256), 0, st, a, part, splits);
  E3_HIP(hipGetLastError());
  return E3_OK;
}
template <class T>
e3_status gated_fwd(const GatedCall& c) {
  constexpr e3_dtype t = std::is_same_v<T, float> ? E3_F32 : E3_BF16;
  GatedArgs a{};
  a.a = {c.x, c.ldx, nullptr, nullptr, 0, (c.M - 1) * c.ldx + c.K};
  a.b = {c.W, 2 * c.N, nullptr, nullptr, 0, c.K * 2 * c.N};
  a.rows = c.M, a.red = c.K, a.cols = (int)c.N, a.bias = c.bias, a.act = c.act, a.y = c.y, a.z = c.z, a.ldy = c.ldy;
  a.ldz = c.ldz, a.gq = c.gq, a.uq = c.uq, a.yq = c.yq, a.gc = c.gc, a.uc = c.uc, a.yc = c.yc;
  a.nt = streams(t, c.M, c.N);
  switch (gated_way(t, c.M, c.K, c.N)) {
    case GatedWay::few: {
      const int splits = gated_few_splits(c.K, c.N);
      a.red_chunk = (int)((c.K + splits - 1) / splits);
      a.part = splits > 1 ? reinterpret_cast<float*>(c.ws) : nullptr;
      {
      TimedLaunch t_("gated_fwd_few", c.st);
      auto* k = c.M == 1 ? k_gated_few<T, 1> : c.M == 2 ? k_gated_few<T, 2> : c.M <= 4 ? k_gated_few<T, 4>
                                                                                   : k_gated_few<T, kGatedFew>;
      hipLaunchKernelGGL(k, dim3((unsigned)((c.N + 31) / 32), (unsigned)splits), dim3(512), 0, c.st, a);
      }
      if (splits > 1) return gated_join<T>(a, a.part, splits, c.st);
      break;
    }
    case GatedWay::panel: return gated_panel<T>(a, c.st);
    case GatedWay::split: {
      // z as a dense layer's partial sums
      using J = Job<T, kAlong, kAcross, kFull, kFull, false>;
      const Cut cut = dense_cut(t, c.M, 2 * c.N, c.K, kForward);
      DenseArgs d{};
      float* part = reinterpret_cast<float*>(c.ws);
      d.a = a.a, d.b = a.b, d.rows = c.M, d.cols = (int)(2 * c.N), d.red = c.K;
      set_cut(d, cut, part);
      const e3_status s = dense_launch<J>(d, cut, {"gated_fwd_split_64", "gated_fwd_split_128", "gated_fwd_split_256"}, c.st);
      if (s != E3_OK) return s;
      return gated_join<T>(a, part, cut.splits, c.st);
    }
    case GatedWay::tile: {
      const int b = dense_cut(t, c.M, 2 * c.N, c.K, kForward).tile;
      if constexpr (t == E3_BF16) {
        // (shorter reductions: two workgroups per CU, one's results stored beside the other's
        // products; 65,536 x 256 to 1,024 with z 131 us so, 138 direct; 16,384 x 512 to 4,096
        // 213 and 191)
        if (b == 256 && c.K >= 512 && c.K % 64 == 0 && direct_side(a.a, 8) && direct_side(a.b, c.N)) {
          using Tl = DirectTile<kAlong, kPaired>;
          TimedLaunch t_("gated_fwd_direct", c.st);
          const int64_t tiles = (c.M + Tl::BM - 1) / Tl::BM * ((c.N + Tl::BN / 2 - 1) / (Tl::BN / 2));
          hipLaunchKernelGGL(k_gated_direct<T>, grid_of(tiles), dim3(Tl::THREADS), 0, c.st, a);
          break;
        }
      }
      TimedLaunch t_(b == 64 ? "gated_fwd_64" : b == 128 ? "gated_fwd_128" : "gated_fwd_256", c.st);
      auto go = [&](auto B) {
        using O = GatedTileOf<T, decltype(B)::value>;
        const int64_t tiles = (c.M + O::BM - 1) / O::BM * ((c.N + O::BN / 2 - 1) / (O::BN / 2));
        hipLaunchKernelGGL((k_gated<T, decltype(B)::value>), grid_of(tiles), dim3(O::THREADS), 0, c.st, a);
      };
      if (b == 64) go(std::integral_constant<int, 64>{});
      else if (b == 128) go(std::integral_constant<int, 128>{});
      else if constexpr (t == E3_BF16) go(std::integral_constant<int, 256>{});
      break;
    }
  }
  E3_HIP(hipGetLastError());
  return E3_OK;
}

}  // namespace
