// What stands before the products of a Muon step: moments, the update's norm, and the update in two fp16 terms.
//
//   muon_moments_kernel   step: m = mu m + (1 - mu) g', U = (1 - mu) g' + mu m (or m); and the sum of U's squares, one partial sum a CTA
//   muon_scale_kernel     X = U 2^k as hi + lo, and what X is to be multiplied by in the first step: 1 / (|U| + eps) is not a power of
//                         two, and U in bf16 is exact in one fp16 term as long as only powers of two touch it
//
// Squares are summed in 64 bits: no update's norm overflows or vanishes.  Bound by the bytes that they move (10 an entry each, of a step).
#include "common.cuh"
#include "muon_kernels.cuh"

#include <cuda_fp16.h>

namespace sffn {
namespace {

constexpr int kThreads = 256;

// Threads of a row of C entries, eight each, at most a CTA's; the others take the next rows.
__device__ __forceinline__ int threads_of_row(int C) {
  int t = 8;
  while (t < kThreads && 8 * t < C) t <<= 1;
  return t;
}

template <int BYTES>
__device__ __forceinline__ bool on(const void* p) { return (reinterpret_cast<uintptr_t>(p) & (BYTES - 1)) == 0; }

__device__ __forceinline__ void load8(const float* p, int count, float* f) {
  if (count == 8 && on<16>(p)) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < count ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int count, float* f) {
  if (count == 8 && on<16>(p)) {
    Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(p), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < count ? __bfloat162float(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void load8(const void* base, bool bf16, int64_t at, int count, float* f) {
  if (bf16) load8(static_cast<const __nv_bfloat16*>(base) + at, count, f);
  else load8(static_cast<const float*>(base) + at, count, f);
}
__device__ __forceinline__ void store8(float* p, int count, const float* f) {
  if (count == 8 && on<16>(p)) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < count) p[i] = f[i];
  }
}

// What a step's gradients are multiplied by; `fine`: whether the step is taken at all.
__device__ __forceinline__ float clip_of(const MuonBatch& b, bool& fine) {
  fine = true;
  if (!b.grad_norm) return 1.f;
  const float norm = *b.grad_norm;
  fine = isfinite(norm);
  return fminf(1.f, b.max_norm / (norm + 1e-6f));
}
// U from the gradient and the moments as this step leaves them.
__device__ __forceinline__ float update_of(const MuonBatch& b, float g, float m) { return b.nesterov ? fmaf(b.momentum, m, b.one_momentum * g) : m; }

template <typename T>
__device__ __forceinline__ T block_sum(T v, T* room) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  T s = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) s += room[w];
  return s;
}

__global__ void __launch_bounds__(kThreads) muon_moments_kernel(const __grid_constant__ MuonBatch b) {
  __shared__ double room[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const MuonItem& it = b.item[blockIdx.y];
  bool fine;
  const float clip = clip_of(b, fine);
  const int per = threads_of_row(b.C), high = kThreads / per;
  double sum = 0.0;
  for (int64_t r = blockIdx.x * high + threadIdx.x / per; r < b.R; r += (int64_t)gridDim.x * high) {
    for (int c = 8 * (threadIdx.x % per); c < b.C; c += 8 * per) {
      const int count = min(8, b.C - c);
      float g[8], m[8];
      load8(it.src, b.src_bf16, r * it.ld_src + c, count, g);
      if (b.step) {
        float* const at = it.m + r * b.C + c;
        load8(at, count, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          g[i] *= clip;
          m[i] = fmaf(b.momentum, m[i], b.one_momentum * g[i]);
          g[i] = update_of(b, g[i], m[i]);
        }
        if (fine) store8(at, count, m);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)g[i], (double)g[i], sum);  // (what is past a row's end is zero)
    }
  }
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) b.squares[blockIdx.y * kMuonPartials + blockIdx.x] = sum;
}

__device__ __forceinline__ uint32_t two_halves(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

__global__ void __launch_bounds__(kThreads) muon_scale_kernel(const __grid_constant__ MuonBatch b, int partials) {
  __shared__ double room[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  static_assert(kMuonPartials <= kThreads, "a partial sum a thread");
  const MuonItem& it = b.item[blockIdx.y];
  const double norm = sqrt(block_sum((int)threadIdx.x < partials ? __ldcg(b.squares + blockIdx.y * kMuonPartials + threadIdx.x) : 0.0, room));
  // as stored: 2^(kMuonExponent - 1) <= norm 2^k < 2^kMuonExponent; a norm that is zero or not finite takes no scale
  const bool some = norm > 0.0 && isfinite(norm);
  const int k = some ? kMuonExponent - 1 - ilogb(norm) : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const double g = some ? scalbn(1.0, kMuonExponent - k) / (norm + (double)b.eps) : norm == 0.0 ? 0.0 : (double)NAN;
    float* const to = b.first + 4 * blockIdx.y;
    to[0] = (float)g;
    to[1] = (float)(g * g);
    to[2] = (float)(g * g * g);
    to[3] = (float)(g * g * g * g * g);
  }
  const double scale = scalbn(1.0, k);
  bool fine;
  const float clip = clip_of(b, fine);
  const int per = threads_of_row(b.C), high = kThreads / per;
  uint16_t* const x = b.x[0] + blockIdx.y * b.x_matrix;
  for (int64_t r = blockIdx.x * high + threadIdx.x / per; r < b.R; r += (int64_t)gridDim.x * high) {
    for (int c = 8 * (threadIdx.x % per); c < b.C; c += 8 * per) {
      const int count = min(8, b.C - c);
      float g[8], m[8];
      load8(it.src, b.src_bf16, r * it.ld_src + c, count, g);
      if (b.step) {
        load8(it.m + r * b.C + c, count, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = update_of(b, g[i] * clip, m[i]);
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[i] = (float)((double)g[i] * scale);
        m[i] = g[i] - __half2float(__float2half_rn(g[i]));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = two_halves(g[2 * i], g[2 * i + 1]);
        lo[i] = two_halves(m[2 * i], m[2 * i + 1]);
      }
      uint16_t* const to = x + r * b.ld_x + c;  // rows end on a multiple of sixteen
      *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(to + b.x_term) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  }
}

// CTAs of a matrix: what fills the device, no more than there are rows for.
int grid_of(const MuonBatch& b, int sm_count) {
  int per = 8;
  while (per < kThreads && 8 * per < b.C) per <<= 1;
  const int high = kThreads / per, rows = (b.R + high - 1) / high, room = (8 * sm_count + b.n - 1) / b.n;
  const int most = room < kMuonPartials ? room : kMuonPartials;
  return rows < most ? rows : most;
}

}  // namespace

cudaError_t launch_muon_moments(const MuonBatch& b, int sm_count, cudaStream_t s) {
  return launch_pdl(muon_moments_kernel, dim3(grid_of(b, sm_count), b.n), dim3(kThreads), 0, s, b);
}
cudaError_t launch_muon_scale(const MuonBatch& b, int sm_count, cudaStream_t s) {
  const int grid = grid_of(b, sm_count);
  return launch_pdl(muon_scale_kernel, dim3(grid, b.n), dim3(kThreads), 0, s, b, grid);
}

}  // namespace sffn
