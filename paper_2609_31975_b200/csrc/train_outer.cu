// Gradients of the weights of a handful of tokens: C[m, n] = sum over k of A[k, m] B[k, n], K small.
//
// Such a product is its own output: 4096 x 14336, one token, writes 352 MB (bf16) for half a flop a byte.  A thread keeps its 16 bytes
// of every row of B in registers and goes down the rows, eight at a time, with the next eight entries of A's rows under way.
// 4096 x 14336, backward pass of 1 / 4 tokens in bf16 155 / 180 us (the tensor-core product: 190, from 5 tokens on no slower);
// 4096 x 8192, 8 / 16 tokens in fp32 276 / 418 us (tiles of FMAs 504 / 654; split for the tensor cores 492 / 495).
#include "train_kernels.cuh"

namespace sffn {
namespace {

constexpr int kThreads = 128, kTall = 8, kRuns = 8;  // threads side by side; rows at a time; times

template <typename T>
struct Most {
  static constexpr int k = sizeof(T) == 2 ? kOuterBf16 : kOuterF32;
};

template <typename T>
__global__ void __launch_bounds__(kThreads) train_outer_kernel(const __grid_constant__ TrainGemm g, int col_ctas, int row_ctas) {
  constexpr int kPer = Elem<T>::kPerVec, kMost = Most<T>::k, kQuads = kTall / kPer > 0 ? kTall / kPer : 1;  // kQuads: 16-byte pieces of eight entries of A
  pdl_launch_dependents();
  pdl_wait();
  const int at_row = blockIdx.x / col_ctas, z = at_row / row_ctas;
  const int n = ((blockIdx.x - at_row * col_ctas) * kThreads + threadIdx.x) * kPer;
  int m = (at_row - z * row_ctas) * (kTall * kRuns);
  if (n >= g.N) return;
  const T* a = static_cast<const T*>(g.a[z].data);  // its rows are a multiple of eight values apart, and as long
  const T* b = static_cast<const T*>(g.b[z].data) + n;
  const int64_t ld_a = g.a[z].ld, ld_b = g.b[z].ld;
  uint4 bv[kMost], av[kMost][kQuads];
#pragma unroll
  for (int k = 0; k < kMost; ++k)
    if (k < g.K) bv[k] = __ldg(reinterpret_cast<const uint4*>(b + k * ld_b));
  auto fetch = [&](int row) {
#pragma unroll
    for (int k = 0; k < kMost; ++k)
      if (k < g.K) {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) av[k][q] = __ldg(reinterpret_cast<const uint4*>(a + k * ld_a + row + q * kPer));
      }
  };
  const int end = min(m + kTall * kRuns, g.M);
  fetch(m);
  T* out = static_cast<T*>(g.epi.out[z]) + n;
  for (; m < end; m += kTall) {
    float2 acc[kTall][kPer / 2];
#pragma unroll
    for (int i = 0; i < kTall; ++i)
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) acc[i][j] = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kMost; ++k) {
      if (k >= g.K) break;
      float af[kTall], bf[kPer];
#pragma unroll
      for (int q = 0; q < kQuads; ++q) Elem<T>::unpack(av[k][q], af + q * kPer);
      Elem<T>::unpack(bv[k], bf);
#pragma unroll
      for (int i = 0; i < kTall; ++i)
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) acc[i][j] = fma2(make_float2(af[i], af[i]), make_float2(bf[2 * j], bf[2 * j + 1]), acc[i][j]);
    }
    if (m + kTall < end) fetch(m + kTall);
#pragma unroll
    for (int i = 0; i < kTall; ++i) {
      if (m + i >= g.M) break;
      uint4 w;
      if constexpr (sizeof(T) == 4) {
        w = make_uint4(__float_as_uint(acc[i][0].x), __float_as_uint(acc[i][0].y), __float_as_uint(acc[i][1].x), __float_as_uint(acc[i][1].y));
      } else {
        uint32_t h[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const __nv_bfloat162 v = __floats2bfloat162_rn(acc[i][q].x, acc[i][q].y);
          h[q] = *reinterpret_cast<const uint32_t*>(&v);
        }
        w = make_uint4(h[0], h[1], h[2], h[3]);
      }
      *reinterpret_cast<uint4*>(out + (m + i) * g.epi.ld_out) = w;
    }
  }
}

template <typename T>
cudaError_t launch(const TrainGemm& g, cudaStream_t s) {
  if (g.K > Most<T>::k) return cudaErrorInvalidValue;
  const int across = kThreads * Elem<T>::kPerVec, down = kTall * kRuns;
  const int col_ctas = (g.N + across - 1) / across, row_ctas = (g.M + down - 1) / down;
  const long long ctas = (long long)col_ctas * row_ctas * g.batch;
  if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_pdl(train_outer_kernel<T>, dim3((unsigned)ctas), dim3(kThreads), 0, s, g, col_ctas, row_ctas);
}

}  // namespace

cudaError_t launch_train_outer(const TrainGemm& g, int dtype, cudaStream_t s) {
  return dtype == SFFN_BF16 ? launch<__nv_bfloat16>(g, s) : launch<float>(g, s);
}

}  // namespace sffn
