// e3mi: the dense layers' large bfloat16 products, operands straight to LDS.
// A unit of its own: the time of the largest register kernels depends on where their code
// lies. 79 KB of k_dense_two, the same bytes 384 KB further into its unit, took 50 us for 43
// (the backward of 100,003 x 16 x 256 bfloat16, silu), 35 for 32 (64 x 128); aligning it to
// 1, 4 or 16 KB moved other kernels by as much to either side.
#include "dense.h"

namespace {

template <class J>
__global__ __launch_bounds__(512, 2) void k_dense_direct(DenseArgs a) {
  using Tl = DirectTile<J::FA, J::FB>;
  static_assert(sizeof(typename J::T) == 2 && J::KA == kFull && J::KB == kFull && !J::SUM);
  __shared__ __align__(16) typename Tl::Buf s0, s1;
  const int64_t tm = (a.rows + Tl::BM - 1) / Tl::BM;
  const int tn = (a.cols + Tl::BN - 1) / Tl::BN;
  int64_t u = block_id();
  if (u >= tm * tn * a.splits) return;
  const int split = (int)(u / (tm * tn));
  u -= split * (tm * tn);
  const TileAt at = tile_at(u, tm, tn);
  const int64_t r0 = at.m * Tl::BM;
  const int c0 = at.n * Tl::BN;
  const int64_t k0 = split * a.chunk, end = k0 + a.chunk < a.red ? k0 + a.chunk : a.red;
  // Without loads between its stores the end waits for none of them (a load's wait is
  // one for every store before it).
  const Tail<typename J::T> tail(a, c0 + Tl::col0() + Rows32<typename J::T, Tl::RN>::col());
  Tl t;
  t.run(s0, s1, a.a, a.b, r0, a.rows, c0, a.cols, k0, end);
  auto* out = Tl::stage(s0, s1);
  auto store = [&](auto bare) {
    each_of([&](auto i) {
      rows32_out<J, Tl::RN, false, decltype(bare)::value>(a, tail, split, r0 + Tl::row0() + 32 * i, c0 + Tl::col0(), k0, end,
                                                          out, t.acc[i]);
    }, std::make_integer_sequence<int, Tl::RM>{});
  };
  if (a.res || a.part) store(std::false_type{});
  else store(std::true_type{});
}

template <Form FA, Form FB>
e3_status direct(const DenseArgs& a, hipStream_t st) {
  using Tl = DirectTile<FA, FB>;
  const int64_t tiles = (a.rows + Tl::BM - 1) / Tl::BM * ((a.cols + Tl::BN - 1) / Tl::BN);
  hipLaunchKernelGGL((k_dense_direct<Job<__bf16, FA, FB, kFull, kFull, false>>), grid_of(tiles * a.splits), dim3(Tl::THREADS), 0,
                     st, a);
  E3_HIP(hipGetLastError());
  return E3_OK;
}

}  // namespace

e3_status dense_direct_fwd(const DenseArgs& a, hipStream_t st) { return direct<kAlong, kAcross>(a, st); }
e3_status dense_direct_dx(const DenseArgs& a, hipStream_t st) { return direct<kAlong, kAlong>(a, st); }
e3_status dense_direct_dw(const DenseArgs& a, hipStream_t st) { return direct<kAcross, kAcross>(a, st); }
