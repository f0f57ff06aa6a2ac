// Tiles that the tensor-core kernels cut along K: adds up their pieces, in the order of K, and does the epilogue.
//
// A CTA has 32 rows x 64 output columns of a tile, a thread four columns of four rows, or 8 rows and one where there are few such CTAs
// (kHidden, which sums 32 rows at a time: 32, and one); sixteen loads of a thread are under way at once.  Bound by the pieces' bytes,
// which are still in L2, and by latency where few tiles have many pieces (1000 tokens, 4096 x 14336: 33 MB of y's pieces, two a tile,
// 10.6 us; 19 MB of z's and u's, 18 a tile, 9.2 us).
#include "train_umma.cuh"

namespace sffn {
namespace {

constexpr int kJoinCols = 64;
__host__ __device__ constexpr int join_threads(int epilogue) { return (epilogue == kEpiHidden ? 32 : 8) * kJoinCols / 4; }

__device__ __forceinline__ void load4(const float* p, float* v, int n) {
  if (n == 4) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float* v, int n) {
  if (n == 4) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
  }
}
// Steps known to the compiler, here and below: of loops to n, inlined three times, nvcc 12.9 drops one, and the first bf16 term of du's
// last columns stayed unstored where four does not divide H (the three calls alone, in a kernel of 20 lines, do the same).
__device__ __forceinline__ void store4(float* p, const float* v, int n) {
  if (n == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* v, int n) {
  if (n == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = __float2bfloat16(v[i]);
  }
}
// Four hidden values as the next products take them: bf16, or three bf16 terms.
template <typename T>
__device__ __forceinline__ void store_hidden(void* base, int64_t at, int64_t limb, const float* v, int n) {
  if (!base) return;
  __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + at;
  store4(p, v, n);
  if constexpr (sizeof(T) == 4) {
    float r[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int l = 1; l < 3; ++l) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] -= __bfloat162float(__float2bfloat16(r[i]));
      store4(p + l * limb, r, n);
    }
  }
}

// kEach: rows of a thread.
template <int EPI, typename T, int kEach>
__global__ void __launch_bounds__(join_threads(EPI)) train_join_kernel(const __grid_constant__ UmmaParams p, int acc_cols, int groups) {
  constexpr bool kFast = sizeof(T) == 2;
  constexpr int kHigh = join_threads(EPI) / (kJoinCols / 4), rows = kHigh * kEach;
  __shared__ float down[EPI == kEpiHidden ? 32 : 1][kJoinCols];
  pdl_launch_dependents();
  const TrainEpilogue& e = p.epi;
  const int across = (p.tile_cols + kJoinCols - 1) / kJoinCols, per = across * groups;  // groups of rows of a tile
  const int t = blockIdx.x / per, in = blockIdx.x - t * per, r0 = in / across * rows, c0 = in % across * kJoinCols;
  const Place at = place_of(p, p.whole + t);
  const int m0 = at.m * kPairRows + r0, n0 = at.n * p.tile_cols + c0;
  if (m0 >= e.M || n0 >= e.N) return;
  pdl_wait();

  const int c = threadIdx.x % (kJoinCols / 4) * 4, r1 = threadIdx.x / (kJoinCols / 4), n = n0 + c;
  float sum_v[kEach][4] = {}, sum_u[EPI == kEpiGateUp ? kEach : 1][4] = {};
  const float* piece = piece_of(p, t) + (size_t)(r0 + r1) * acc_cols + c0 + c;
  const size_t next = (p.tiles - p.whole) * p.piece;  // from a tile's piece to its next one
#pragma unroll (EPI == kEpiGateUp ? 8 / kEach : 16 / kEach)
  for (int q = 0; q < p.split; ++q, piece += next) {
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
      if (m0 + r1 + x * kHigh >= e.M) continue;  // rows that no pair has written
      const float4 f = __ldcg(reinterpret_cast<const float4*>(piece + (size_t)x * kHigh * acc_cols));
      sum_v[x][0] += f.x; sum_v[x][1] += f.y; sum_v[x][2] += f.z; sum_v[x][3] += f.w;
      if constexpr (EPI == kEpiGateUp) {
        const float4 g = __ldcg(reinterpret_cast<const float4*>(piece + (size_t)x * kHigh * acc_cols + 128));
        sum_u[x][0] += g.x; sum_u[x][1] += g.y; sum_u[x][2] += g.z; sum_u[x][3] += g.w;
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kEach; ++x) {
    const int r = r1 + x * kHigh, m = m0 + r;
    const int left = m < e.M ? min(4, e.N - n) : 0;
    float (&v)[4] = sum_v[x];
    float (&u)[4] = sum_u[EPI == kEpiGateUp ? x : 0];
    if constexpr (EPI == kEpiStore) {
      if (left > 0) store4(static_cast<T*>(e.out[at.batch]) + m * e.ld_out + n, v, left);
    } else if constexpr (EPI == kEpiGateUp) {
      if (left <= 0) continue;
      float h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e.bias && j < left) v[j] += e.bias[n + j];
        h[j] = train_act<kFast>(e.act, v[j]) * train_act<kFast>(e.act_up, u[j]);
      }
      if (e.z) {
        store4(static_cast<T*>(e.z) + m * e.ld_zu + n, v, left);
        store4(static_cast<T*>(e.u) + m * e.ld_zu + n, u, left);
      }
      store_hidden<T>(e.h, m * e.ld_h + n, e.limb, h, left);
    } else {
      float du[4] = {}, h[4];
      if (left > 0) {
        float zv[4];
        load4(static_cast<const T*>(e.z) + m * e.ld_zu + n, zv, left);
        load4(static_cast<const T*>(e.u) + m * e.ld_zu + n, u, left);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float a, da, b, db;
          train_act_slope<kFast>(e.act, zv[j], a, da);
          train_act_slope<kFast>(e.act_up, u[j], b, db);
          h[j] = a * b;
          du[j] = v[j] * a * db;
          v[j] = v[j] * b * da;
        }
        store_hidden<T>(e.dz, m * e.ld_h + n, e.limb, v, left);
        store_hidden<T>(e.du, m * e.ld_h + n, e.limb, du, left);
        store_hidden<T>(e.h, m * e.ld_h + n, e.limb, h, left);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) down[r][c + j] = j < left ? v[j] : 0.f;
    }
  }
  if (EPI == kEpiHidden && e.db) {
    __syncthreads();
    const int n = n0 + threadIdx.x;
    if (threadIdx.x < kJoinCols && n < e.N) {
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 32; ++r) sum += down[r][threadIdx.x];
      e.db[(int64_t)(m0 >> 5) * e.ld_h + n] = sum;
    }
  }
}

template <int EPI, typename T, int kEach>
cudaError_t launch(const UmmaParams& p, cudaStream_t s) {
  const int across = (p.tile_cols + kJoinCols - 1) / kJoinCols, cols = piece_cols(EPI, sizeof(T) == 4), rows = join_threads(EPI) / (kJoinCols / 4) * kEach;
  const int tall = p.m_tiles > 1 || p.epi.M > kPairRows ? kPairRows : p.epi.M, groups = (tall + rows - 1) / rows;
  return launch_pdl(train_join_kernel<EPI, T, kEach>, dim3((unsigned)((p.tiles - p.whole) * across * groups)), dim3(join_threads(EPI)), 0, s, p, cols, groups);
}
template <typename T>
cudaError_t launch(const UmmaParams& p, int epilogue, cudaStream_t s) {
  const bool many = (long long)(p.tiles - p.whole) * p.tile_cols / kJoinCols >= 148;
  if (epilogue == kEpiStore) return many ? launch<kEpiStore, T, 4>(p, s) : launch<kEpiStore, T, 1>(p, s);
  if (epilogue == kEpiGateUp) return many ? launch<kEpiGateUp, T, 4>(p, s) : launch<kEpiGateUp, T, 1>(p, s);
  return launch<kEpiHidden, T, 1>(p, s);
}

}  // namespace

cudaError_t launch_train_join(const UmmaParams& p, int epilogue, bool f32, cudaStream_t s) {
  return f32 ? launch<float>(p, epilogue, s) : launch<__nv_bfloat16>(p, epilogue, s);
}

}  // namespace sffn
