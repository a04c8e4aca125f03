// Shared by the invariant layers (dense.hip, norm.hip): element types, row
// access, activations and the 8-bit checkpoint format.
#pragma once
#include "e3mi_impl.h"

namespace {

typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef unsigned u2v __attribute__((ext_vector_type(2)));
typedef unsigned u4v __attribute__((ext_vector_type(4)));

// i / n of block-uniformly small i by a 32-bit division, a few times cheaper.
__device__ __forceinline__ int64_t div_small(int64_t i, int64_t n) {
  return block_id() < (1 << 23) && n < (1 << 30) ? (int64_t)((unsigned)i / (unsigned)n) : i / n;
}

// ------------------------------------------------------------ element types
// A lane's piece of a row is 16 bytes: V values of the type.  Rows start at
// any element (odd widths, slices of wider tensors), so the vector types claim
// an element's alignment only; the loads are 16-byte instructions either way.
template <class T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int V = 4;
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void get(vec u, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = u[i];
  }
  static __device__ __forceinline__ vec put(const float (&v)[4]) { return vec{v[0], v[1], v[2], v[3]}; }
  static __device__ __forceinline__ float one(float u) { return u; }
  static __device__ __forceinline__ float round(float v) { return v; }
};
template <>
struct Elem<__bf16> {
  static constexpr int V = 8;
  typedef unsigned vec __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void get(vec u, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ vec put(const float (&v)[8]) {
    vec u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(f2v{v[2 * i], v[2 * i + 1]}, bf2v));
    return u;
  }
  static __device__ __forceinline__ float one(__bf16 u) { return (float)u; }
  static __device__ __forceinline__ float round(float v) { return (float)(__bf16)v; }
};

// The values at p (n of them inside the row; the rest read as zero).
template <class T>
__device__ __forceinline__ void ld_piece(const T* p, int n, float (&v)[Elem<T>::V]) {
  if (n >= Elem<T>::V) {
    Elem<T>::get(*reinterpret_cast<const typename Elem<T>::vec*>(p), v);
  } else {
#pragma unroll
    for (int i = 0; i < Elem<T>::V; ++i) v[i] = i < n ? Elem<T>::one(p[i]) : 0.0f;
  }
}
// The same as they lie in memory.
template <class T>
__device__ __forceinline__ typename Elem<T>::vec ld_raw(const T* p, int n) {
  if (n >= Elem<T>::V) return *reinterpret_cast<const typename Elem<T>::vec*>(p);
  if (n <= 0) return typename Elem<T>::vec{};
  float v[Elem<T>::V];
#pragma unroll
  for (int i = 0; i < Elem<T>::V; ++i) v[i] = i < n ? Elem<T>::one(p[i]) : 0.0f;
  return Elem<T>::put(v);
}
// The 16, 8 or 4 bytes r moved down by `bits`, zeros from above; its lowest bits.
__device__ __forceinline__ u4v shift_down(u4v r, unsigned bits) {
  uint64_t lo = (uint64_t)r.y << 32 | r.x, hi = (uint64_t)r.w << 32 | r.z;
  if (bits & 64) lo = hi, hi = 0;
  const unsigned b = bits & 63;
  lo = b ? lo >> b | hi << (64 - b) : lo;
  hi >>= b;
  if (bits >= 128) lo = hi = 0;
  return u4v{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}
__device__ __forceinline__ u2v shift_down(u2v r, unsigned bits) {
  const uint64_t v = bits < 64 ? ((uint64_t)r.y << 32 | r.x) >> bits : 0;
  return u2v{(unsigned)v, (unsigned)(v >> 32)};
}
__device__ __forceinline__ unsigned shift_down(unsigned r, unsigned bits) { return bits < 32 ? r >> bits : 0u; }
__device__ __forceinline__ unsigned low_bits(unsigned r, int bits) {
  return bits >= 32 ? r : bits <= 0 ? 0u : r & ~(~0u << bits);
}
__device__ __forceinline__ u2v low_bits(u2v r, int bits) { return u2v{low_bits(r.x, bits), low_bits(r.y, bits - 32)}; }
__device__ __forceinline__ u4v low_bits(u4v r, int bits) {
  return u4v{low_bits(r.x, bits), low_bits(r.y, bits - 32), low_bits(r.z, bits - 64), low_bits(r.w, bits - 96)};
}
// Values at .. at + n - 1 of a matrix that spans `total` values from p, the rest
// of the piece zero, without a branch, so that several loads are in flight: a
// piece that would reach past the span is loaded from its last values and moved
// down.  total is at least a piece.  The load and its cutting are apart: cutting
// waits for the load.
struct Cutting {
  unsigned down_keep;  // bits to move down << 16 | bits to keep
  template <class R>
  __device__ __forceinline__ R operator()(R r) const {
    return low_bits(shift_down(r, down_keep >> 16), (int)(down_keep & 0xffffu));
  }
  __device__ __forceinline__ bool none() const { return (down_keep & 0xffffu) == 0; }
};
template <class R, class E>
__device__ __forceinline__ R ld_span(const E* p, int64_t at, int64_t total, int n, Cutting& cut) {
  typedef R Any __attribute__((aligned(sizeof(E))));
  constexpr int V = sizeof(R) / sizeof(E), BITS = 8 * sizeof(E);
  const int64_t start = at < total - V ? at : total - V, over = at - start;
  cut.down_keep = (over < V ? (unsigned)over : (unsigned)V) * BITS << 16 | (unsigned)(n * BITS);
  return *reinterpret_cast<const Any*>(p + start);
}
// nt: past the caches, for outputs that do not fit them (rule and figures at
// streams()).
template <class T>
__device__ __forceinline__ void st_piece(T* p, int n, const float (&v)[Elem<T>::V], bool nt = false) {
  if (n >= Elem<T>::V) {
    auto* q = reinterpret_cast<typename Elem<T>::vec*>(p);
    if (nt) {
      asm volatile("");  // keeps the two stores apart: the compiler would merge them into an ordinary one
      __builtin_nontemporal_store(Elem<T>::put(v), q);
      asm volatile("");
    } else {
      *q = Elem<T>::put(v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < Elem<T>::V; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

// ------------------------------------------------------------ sums over lanes
// Over aligned groups of L lanes (a power of two up to 64); every lane of a
// group ends with the same bits.  All lanes of the group take part.
template <int CTRL>
__device__ __forceinline__ unsigned dpp_u(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int L, class F>
__device__ __forceinline__ unsigned fold_lanes(unsigned v, F&& f) {
  if constexpr (L >= 2) v = f(v, dpp_u<0xb1>(v));   // quad_perm [1, 0, 3, 2]
  if constexpr (L >= 4) v = f(v, dpp_u<0x4e>(v));   // quad_perm [2, 3, 0, 1]
  if constexpr (L >= 8) v = f(v, dpp_u<0x141>(v));  // row_half_mirror
  if constexpr (L >= 16) v = f(v, dpp_u<0x140>(v)); // row_mirror
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(r[0], r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = f(r[0], r[1]);
  }
  return v;
}
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
  return __uint_as_float(fold_lanes<L>(__float_as_uint(v), [](unsigned a, unsigned b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
// Over the lanes of the wave that are congruent modulo C (4 or 8).
template <int C>
__device__ __forceinline__ float sum_strided(float v) {
  static_assert(C == 4 || C == 8);
  auto add = [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); };
  unsigned u = __float_as_uint(v);
  if constexpr (C == 4) u = add(u, dpp_u<0x124>(u));  // row_ror:4
  u = add(u, dpp_u<0x128>(u));                        // row_ror:8
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  u = add(r[0], r[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(add(q[0], q[1]));
}
template <int L>
__device__ __forceinline__ unsigned max_lanes(unsigned v) {
  return fold_lanes<L>(v, [](unsigned a, unsigned b) { return a > b ? a : b; });
}

// ------------------------------------------------------------ 8-bit checkpoints
// Groups of 32 values along a row share the power of two 2^(c - 127) and hold
// integers q of [-127, 127].  c - 127 = floor(log2 max|x|) - 6, one more where
// the largest would round past 127, at least -127; q = x 2^(127 - c) to
// nearest, ties to even.  The product by a power of two is exact, so a value is
// off by at most half a step.  The step stays at 2^121 at the range's end, where
// 64 of the next would be infinite: values from 127.5 of it on read as 127.  An
// infinity or a NaN in the group makes all of it NaN (c = 255, q = 0).
constexpr int kGroup = 32;

__device__ __forceinline__ float step8(unsigned c) {
  return __uint_as_float(c == 255u ? 0x7fc00000u : c == 0u ? 0x00400000u : c << 23);
}
// The group's exponent byte from its largest magnitude's bits (NaN above all).
__device__ __forceinline__ unsigned exp8(unsigned top) {
  if (top >= 0x7f800000u) return 255u;
  const int e = (int)((top + 0x10000u) >> 23) - 6;  // 1.1111111 and more in binary carries
  return e < 0 ? 0u : e > 248 ? 248u : (unsigned)e;
}
template <int V>
struct Bytes;
template <>
struct Bytes<4> {
  typedef unsigned vec __attribute__((aligned(1)));
};
template <>
struct Bytes<8> {
  typedef u2v vec __attribute__((aligned(1)));
};

// Packs a lane's V values at column col of a row (n of them inside it); the
// 32 / V lanes of a group hold consecutive pieces and all take part.  q and c
// point at the row.
template <int V>
__device__ __forceinline__ void pack8_piece(const float (&v)[V], int col, int n, int8_t* q, uint8_t* c) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const unsigned b = i < n ? __float_as_uint(v[i]) & 0x7fffffffu : 0u;
    top = b > top ? b : top;
  }
  top = max_lanes<kGroup / V>(top);
  if (n <= 0) return;
  const unsigned e = exp8(top);
  const float up = e == 255u ? 0.0f : __uint_as_float((254u - e) << 23);
  unsigned w[V / 4];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int k = e == 255u ? 0 : (int)fminf(fmaxf(rintf(v[i] * up), -127.0f), 127.0f);
    if (i % 4 == 0) w[i / 4] = 0;
    w[i / 4] |= ((unsigned)k & 0xffu) << (8 * (i % 4));
  }
  if (n >= V) {
    if constexpr (V == 4) *reinterpret_cast<typename Bytes<4>::vec*>(q + col) = w[0];
    else *reinterpret_cast<typename Bytes<8>::vec*>(q + col) = u2v{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) q[col + i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  if (col % kGroup == 0) c[col / kGroup] = (uint8_t)e;
}

// V packed values at column col of a row (n inside it; the rest zero) and their
// group's exponent byte, as they lie in memory.
template <int V>
struct Raw8 {
  unsigned w[V / 4];
  unsigned e;
};
template <int V>
__device__ __forceinline__ Raw8<V> ld_raw8(const int8_t* q, const uint8_t* c, int col, int n) {
  Raw8<V> r{};
  if (n <= 0) return r;
  r.e = c[col / kGroup];
  if (n >= V) {
    if constexpr (V == 4) {
      r.w[0] = *reinterpret_cast<const typename Bytes<4>::vec*>(q + col);
    } else {
      const u2v t = *reinterpret_cast<const typename Bytes<8>::vec*>(q + col);
      r.w[0] = t.x, r.w[1] = t.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) r.w[i / 4] |= ((unsigned)(uint8_t)q[col + i]) << (8 * (i % 4));
  }
  return r;
}
template <int V>
__device__ __forceinline__ void get8(const Raw8<V>& r, float (&v)[V]) {
  const float s = step8(r.e);
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (float)(int)(int8_t)(r.w[i / 4] >> (8 * (i % 4))) * s;
}

// Values of a row that is kept in full or packed (x null).
template <class T>
struct RowsIn {
  const T* x;
  int64_t ld;
  const int8_t* q;
  const uint8_t* c;
  // One of the two, known at compile time, as it lies in memory.
  template <bool Q>
  using Raw = typename std::conditional<Q, Raw8<Elem<T>::V>, typename Elem<T>::vec>::type;
  template <bool Q>
  __device__ __forceinline__ Raw<Q> raw(int64_t row, int col, int cols) const {
    if constexpr (Q) return ld_raw8<Elem<T>::V>(q + row * cols, c + row * ((cols + kGroup - 1) / kGroup), col, cols - col);
    else return ld_raw<T>(x + row * ld + col, cols - col);
  }
  template <bool Q>
  static __device__ __forceinline__ void get(const Raw<Q>& r, float (&v)[Elem<T>::V]) {
    if constexpr (Q) get8(r, v);
    else Elem<T>::get(r, v);
  }
  __device__ __forceinline__ void load(int64_t row, int col, int cols, float (&v)[Elem<T>::V]) const {
    if (x) get<false>(raw<false>(row, col, cols), v);
    else get<true>(raw<true>(row, col, cols), v);
  }
  __device__ __forceinline__ float value(int64_t row, int col, int cols) const {
    if (x) return Elem<T>::one(x[row * ld + col]);
    return (float)q[row * cols + col] * step8(c[row * ((cols + kGroup - 1) / kGroup) + col / kGroup]);
  }
};

// ------------------------------------------------------------ activations
// gelu is z Phi(z) with the normal distribution's Phi.  The library's erf and exp
// took a third of a wide layer's forward; one hardware exponential serves both
// Phi and its density:
//   Phi(-a) = exp(-a^2 / 2) G(1 / (1 + 0.35 a)) for a >= 0, G a polynomial of
//   degree 9 fitted to the smallest relative error over a <= 14 (2.7e-8),
// computed in float32.  The exponential's argument is rounded, so that gelu's
// relative error grows with its tail: 1.5e-6 where z > -5, 2.8e-6 where z > -8 (and
// gelu is 5e-15), 7.5e-6 where z > -12; 4e-7 for z > 0.  silu's likewise: 4e-7 where
// z > -5, 9e-7 where z > -12, 4e-6 where z > -80.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float a = __builtin_fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
  constexpr float C[10] = {-1.886859763544635e-06f, 0.13966286182403564f,   0.13947750627994537f,
                           0.12180975824594498f,    0.09927769750356674f,   -0.010595494881272316f,
                           0.14310124516487122f,    -0.24294354021549225f,  0.13825730979442596f,
                           -0.028045475482940674f};
  float g = C[9];
#pragma unroll
  for (int i = 8; i >= 0; --i) g = fmaf(g, t, C[i]);
  e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);  // exp(-z^2 / 2)
  const float tail = e * g;
  return z > 0.0f ? 1.0f - tail : tail;
}
__device__ __forceinline__ float sigmoid(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}
__device__ __forceinline__ float act_of(int act, float z) {
  if (act == E3_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if (act == E3_ACT_SILU) return z * sigmoid(z);
  if (act == E3_ACT_GELU) {
    float e;
    return z * normal_cdf(z, e);
  }
  return z;
}
__device__ __forceinline__ float act_grad(int act, float z) {
  if (act == E3_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  if (act == E3_ACT_SILU) {
    const float s = sigmoid(z);
    return s * (1.0f + z * (1.0f - s));
  }
  if (act == E3_ACT_GELU) {
    float e;
    const float p = normal_cdf(z, e);
    return fmaf(z * 0.39894228f, e, p);
  }
  return 1.0f;
}
// Over a piece: one branch on the (uniform) activation for all values.
template <int V>
__device__ __forceinline__ void act_piece(int act, float (&v)[V]) {
  if (act == E3_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_of(E3_ACT_SILU, v[i]);
  } else if (act == E3_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_of(E3_ACT_GELU, v[i]);
  } else if (act == E3_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_of(E3_ACT_RELU, v[i]);
  }
}
// v act'(z).
template <int V>
__device__ __forceinline__ void act_grad_piece(int act, const float (&z)[V], float (&v)[V]) {
  if (act == E3_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= act_grad(E3_ACT_SILU, z[i]);
  } else if (act == E3_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= act_grad(E3_ACT_GELU, z[i]);
  } else if (act == E3_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= act_grad(E3_ACT_RELU, z[i]);
  }
}

// ------------------------------------------------------------ column sums
// Sums over p of part[p pitch + c], c < n0 to out0 and n0 <= c < n to out1
// (either may be null), in a fixed order: 32 threads of a column take every 32nd
// partial in eight running sums (16 columns' loads are in flight together:
// latency is all there is to it), then their sums are added in order.
template <class T>
__global__ __launch_bounds__(512) void k_column_sums(const float* part, int parts, int64_t pitch, int64_t n0, int64_t n,
                                                     T* out0, T* out1) {
  __shared__ float s[32][17];
  const int c = threadIdx.x % 16, p0 = threadIdx.x / 16;
  const int64_t first = block_id() * 16, col = first + c;
  if (first >= n || (!out0 && first + 16 <= n0) || (!out1 && first >= n0)) return;
  float t[8] = {};
  if (col < n)
    for (int p = p0; p < parts; p += 256)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p + 32 * i < parts) t[i] += part[(p + 32 * i) * pitch + col];
  s[p0][c] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
  __syncthreads();
  if (p0 != 0 || col >= n) return;
  float v = 0.0f;
#pragma unroll
  for (int p = 0; p < 32; ++p) v += s[p][c];
  T* out = col < n0 ? out0 + col : out1 + (col - n0);
  if (col < n0 ? out0 != nullptr : out1 != nullptr) *out = (T)v;
}

inline e3_status column_sums(e3_dtype dtype, const float* part, int parts, int64_t pitch, int64_t n0, int64_t n,
                             void* out0, void* out1, hipStream_t st) {
  TimedLaunch t_("column_sums", st);
  const dim3 grid = grid_of((n + 15) / 16);
  if (dtype == E3_F32)
    hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(512), 0, st, part, parts, pitch, n0, n,
                       static_cast<float*>(out0), static_cast<float*>(out1));
  else
    hipLaunchKernelGGL(k_column_sums<__bf16>, grid, dim3(512), 0, st, part, parts, pitch, n0, n,
                       static_cast<__bf16*>(out0), static_cast<__bf16*>(out1));
  E3_HIP(hipGetLastError());
  return E3_OK;
}

// Whether an output of this size is written with non-temporal stores: when it
// exceeds the second-level caches (8 x 4 MB), so that whoever reads it next does
// not find it there anyway.  Against ordinary stores: 1,248,000 x 8 x 64 float32 62 us
// (129), 1,248,000 x 64 x 64 137 (207), bfloat16 59 (78); 156,000 x 64 x 1,664 278
// (498), bfloat16 121 (228).
inline bool streams(e3_dtype t, int64_t rows, int64_t cols) { return rows * cols * (t == E3_F32 ? 4 : 2) > (32 << 20); }

// ------------------------------------------------------------ argument checks
constexpr int64_t kMaxCols = 1 << 20;               // widths; a row's offsets stay in 32 bits
constexpr int64_t kMaxRows = (int64_t)1 << 40;
inline bool good_dtype(e3_dtype t) { return t == E3_F32 || t == E3_BF16; }
inline bool good_rows(e3_dtype t, int64_t rows, int64_t cols) {
  return good_dtype(t) && rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxCols;
}
inline bool misaligned(e3_dtype t, const void* p) {
  return reinterpret_cast<uintptr_t>(p) & (t == E3_F32 ? 3u : 1u);
}
inline bool good_ptr(e3_dtype t, const void* p) { return p && !misaligned(t, p); }

}  // namespace
