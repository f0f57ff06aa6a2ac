// Products of the training calls on the CUDA cores: fp32 FMAs, operands fp32 or bf16, any size and either order of the
// operands in memory.  One CTA owns a 64 x 64 tile, a thread 4 x 4 of it.
#include "train_kernels.cuh"

namespace sffn {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// A [kDepth][kTile] piece of an operand, zeros outside of it.
template <typename T>
__device__ __forceinline__ void fetch(float (*s)[kTile + 4], const TrainOperand& o, bool major_k, int row0, int rows, int k0, int K) {
  const T* p = static_cast<const T*>(o.data);
  for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
    const int r = major_k ? i / kDepth : i % kTile, k = major_k ? i % kDepth : i / kTile;
    float v = 0.f;
    if (row0 + r < rows && k0 + k < K) v = value_of(p[major_k ? (int64_t)(row0 + r) * o.ld + k0 + k : (int64_t)(k0 + k) * o.ld + row0 + r]);
    s[k][r] = v;
  }
}

template <typename T, int EPI>
__global__ void __launch_bounds__(kThreads) train_simt_kernel(const __grid_constant__ TrainGemm g) {
  constexpr int kSums = EPI == kEpiGateUp ? 2 : 1;
  constexpr bool kFast = sizeof(T) == 2;
  __shared__ float sa[kDepth][kTile + 4], sb[kSums][kDepth][kTile + 4];
  __shared__ float column[EPI == kEpiHidden ? 16 : 1][kTile];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile, z = blockIdx.z;
  float acc[kSums][4][4] = {};
  const int parts = EPI == kEpiGateUp ? 1 : g.parts;
  for (int part = 0; part < parts; ++part) {
    const int at = g.batch > 1 ? z : part;
    for (int k0 = 0; k0 < g.K; k0 += kDepth) {
      fetch<T>(sa, g.a[at], g.a_major_k, m0, g.M, k0, g.K);
#pragma unroll
      for (int q = 0; q < kSums; ++q) fetch<T>(sb[q], g.b[kSums > 1 ? q : at], g.b_major_k, n0, g.N, k0, g.K);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kDepth; ++k) {
        const float4 a = *reinterpret_cast<const float4*>(&sa[k][4 * ty]);
        const float av[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int q = 0; q < kSums; ++q) {
          const float4 b = *reinterpret_cast<const float4*>(&sb[q][k][4 * tx]);
          const float bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[q][i][j] = fmaf(av[i], bv[j], acc[q][i][j]);
        }
      }
      __syncthreads();
    }
  }
  const TrainEpilogue& e = g.epi;
  float down[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 4 * ty + i;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + 4 * tx + j;
      if (m >= g.M || n >= g.N) continue;
      if (EPI == kEpiStore) {
        put(static_cast<T*>(e.out[z]) + m * e.ld_out + n, acc[0][i][j]);
      } else if (EPI == kEpiGateUp) {
        const float zv = acc[0][i][j] + (e.bias ? e.bias[n] : 0.f), uv = acc[kSums - 1][i][j];
        if (e.z) {
          put(static_cast<T*>(e.z) + m * e.ld_zu + n, zv);
          put(static_cast<T*>(e.u) + m * e.ld_zu + n, uv);
        }
        put(static_cast<T*>(e.h) + m * e.ld_h + n, train_act<kFast>(e.act, zv) * train_act<kFast>(e.act_up, uv));
      } else {
        const float zv = value_of(static_cast<const T*>(e.z)[m * e.ld_zu + n]), uv = value_of(static_cast<const T*>(e.u)[m * e.ld_zu + n]);
        float a, da, b, db;
        train_act_slope<kFast>(e.act, zv, a, da);
        train_act_slope<kFast>(e.act_up, uv, b, db);
        const float dz = acc[0][i][j] * b * da, du = acc[0][i][j] * a * db;
        if (e.dz) put(static_cast<T*>(e.dz) + m * e.ld_h + n, dz);
        if (e.du) put(static_cast<T*>(e.du) + m * e.ld_h + n, du);
        if (e.h) put(static_cast<T*>(e.h) + m * e.ld_h + n, a * b);
        down[j] += dz;
      }
    }
  }
  if (EPI == kEpiHidden && e.db) {
#pragma unroll
    for (int j = 0; j < 4; ++j) column[ty][4 * tx + j] = down[j];
    __syncthreads();
    if (threadIdx.x < kTile && n0 + threadIdx.x < g.N) {
      float sum = 0.f;
      for (int r = 0; r < 16; ++r) sum += column[r][threadIdx.x];
      e.db[blockIdx.y * e.ld_h + n0 + threadIdx.x] = sum;
    }
  }
}

__global__ void __launch_bounds__(256) column_sums_kernel(const float* partial, int lines, int64_t ld, int N, float* out) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  float sum = 0.f;
  for (int l = 0; l < lines; ++l) sum += partial[l * ld + n];
  out[n] = sum;
}

template <typename T>
cudaError_t launch(const TrainGemm& g, cudaStream_t s) {
  const dim3 grid((g.N + kTile - 1) / kTile, (g.M + kTile - 1) / kTile, g.batch > 1 ? g.batch : 1);
  if (g.epilogue == kEpiStore) train_simt_kernel<T, kEpiStore><<<grid, kThreads, 0, s>>>(g);
  else if (g.epilogue == kEpiGateUp) train_simt_kernel<T, kEpiGateUp><<<grid, kThreads, 0, s>>>(g);
  else train_simt_kernel<T, kEpiHidden><<<grid, kThreads, 0, s>>>(g);
  return cudaGetLastError();
}

}  // namespace

int train_simt_lines(int M) { return (M + kTile - 1) / kTile; }

cudaError_t launch_train_simt(const TrainGemm& g, int dtype, cudaStream_t s) {
  return dtype == SFFN_BF16 ? launch<__nv_bfloat16>(g, s) : launch<float>(g, s);
}

cudaError_t launch_train_column_sums(const float* partial, int lines, int64_t ld, int N, float* out, cudaStream_t s) {
  column_sums_kernel<<<(N + 255) / 256, 256, 0, s>>>(partial, lines, ld, N, out);
  return cudaGetLastError();
}

}  // namespace sffn
