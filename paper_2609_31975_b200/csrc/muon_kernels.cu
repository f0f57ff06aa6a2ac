// What stands before the products of a Muon step: moments, the update's norm, and the update in two fp16 terms.
//
//   muon_moments_kernel   step: m = mu m + (1 - mu) g', U = (1 - mu) g' + mu m (or m); and the sum of U's squares, one partial sum a CTA
//   muon_scale_kernel     X = U 2^k as hi + lo, and what X is to be multiplied by in the first step: 1 / (|U| + eps) is not a power of
//                         two, and U in bf16 is exact in one fp16 term as long as only powers of two touch it
//
// Squares are summed in 64 bits: no update's norm overflows or vanishes.  Both are bound by the bytes that they move, so several turns' loads
// are under way at once, from four CTAs an SM.  A step of 14336 x 4096 with bf16 gradients (10 bytes an entry each): moments 94 us, X 99 us,
// 6.2 and 5.9 TB/s (one turn at a time, 256 CTAs: 162 and 172).  Orthogonalisation of 14230 x 3840, bf16: 26 us (109 MB, 4.2 TB/s) and 54 us
// (327 MB, 6.1 TB/s); 75 and 102 before.
#include "common.cuh"
#include "muon_kernels.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace sffn {
namespace {

constexpr int kThreads = 256, kCtas = 4;  // CTAs of an SM, all of a launch at once

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
// The same of a matrix in bf16 or fp32.  Eight bf16 stay as they came (true) until entries() is called: to unpack them is to wait for them.
__device__ __forceinline__ bool load8(const void* base, bool bf16, int64_t at, int count, float* f) {
  if (!bf16) {
    load8(static_cast<const float*>(base) + at, count, f);
    return false;
  }
  const __nv_bfloat16* const p = static_cast<const __nv_bfloat16*>(base) + at;
  const bool packed = count == 8 && on<16>(p);
  if (packed) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < count ? __bfloat162float(p[i]) : 0.f;
  }
  return packed;
}
__device__ __forceinline__ void entries(bool packed, float* f) {
  if (packed) Elem<__nv_bfloat16>::unpack(make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])), f);
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

// Eight entries a turn and kAhead turns at a time, all of which are loaded before the first is used: `use(row, column, count, entries, moments)`.
template <bool STEP>
constexpr int kAhead = STEP ? 2 : 4;
template <bool STEP, typename Use>
__device__ __forceinline__ void for_entries(const MuonBatch& b, const MuonItem& it, const Use& use) {
  constexpr int kA = kAhead<STEP>;
  const int per = threads_of_row(b.C), high = kThreads / per, c0 = 8 * (threadIdx.x % per);
  const int64_t stride = (int64_t)gridDim.x * high;
  int64_t r[kA];
  int c[kA];
  bool packed[kA];
  int64_t row = blockIdx.x * high + threadIdx.x / per;
  int column = c0;
  while (row < b.R && column < b.C) {
    float g[kA][8], m[STEP ? kA : 1][8];
#pragma unroll
    for (int a = 0; a < kA; ++a) {
      r[a] = row;
      c[a] = column;
      if (row < b.R) {
        packed[a] = load8(it.src, b.src_bf16, row * it.ld_src + column, min(8, b.C - column), g[a]);
        if (STEP) load8(it.m + row * b.C + column, min(8, b.C - column), m[a]);
        column += 8 * per;
        if (column >= b.C) {
          column = c0;
          row += stride;
        }
      }
    }
#pragma unroll
    for (int a = 0; a < kA; ++a)
      if (r[a] < b.R) {
        entries(packed[a], g[a]);
        use(r[a], c[a], min(8, b.C - c[a]), g[a], m[STEP ? a : 0]);
      }
  }
}

template <bool STEP>
__global__ void __launch_bounds__(kThreads, kCtas) muon_moments_kernel(const __grid_constant__ MuonBatch b) {
  __shared__ double room[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const MuonItem& it = b.item[blockIdx.y];
  bool fine;
  const float clip = clip_of(b, fine);
  double sum = 0.0;
  for_entries<STEP>(b, it, [&](int64_t r, int c, int count, float* g, float* m) {
    if (STEP) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[i] *= clip;
        m[i] = fmaf(b.momentum, m[i], b.one_momentum * g[i]);
        g[i] = update_of(b, g[i], m[i]);
      }
      if (fine) store8(it.m + r * b.C + c, count, m);
    }
    // eight squares in fp32, where they fit (conversions to 64 bits are slow), and in 64 bits from there on; what is past a row's end is zero
    float eight = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) eight = fmaf(g[i], g[i], eight);
    if (eight >= 0x1p-100f && eight <= 0x1p125f) {
      sum += (double)eight;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fma((double)g[i], (double)g[i], sum);
    }
  });
  sum = block_sum(sum, room);
  if (threadIdx.x == 0) b.squares[blockIdx.y * kMuonPartials + blockIdx.x] = sum;
}

__device__ __forceinline__ uint32_t two_halves(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <bool STEP>
__global__ void __launch_bounds__(kThreads, kCtas) muon_scale_kernel(const __grid_constant__ MuonBatch b, int partials) {
  __shared__ double room[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const MuonItem& it = b.item[blockIdx.y];
  double sum = 0.0;
  for (int i = threadIdx.x; i < partials; i += kThreads) sum += __ldcg(b.squares + blockIdx.y * kMuonPartials + i);
  const double norm = sqrt(block_sum(sum, room));
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
  // 2^k in two factors, as k may be 162; both products are exact, or smaller than anything that fp16 holds
  const float half = scalbnf(1.f, k / 2), rest = scalbnf(1.f, k - k / 2);
  bool fine;
  const float clip = clip_of(b, fine);
  uint16_t* const x = b.x[0] + blockIdx.y * b.x_matrix;
  for_entries<STEP>(b, it, [&](int64_t r, int c, int, float* g, float* m) {
    if (STEP) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = update_of(b, g[i] * clip, m[i]);
    }
    uint32_t hi[4], lo[4];
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] = g[i] * half * rest;
      left[i] = g[i] - __half2float(__float2half_rn(g[i]));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = two_halves(g[2 * i], g[2 * i + 1]);
      lo[i] = two_halves(left[2 * i], left[2 * i + 1]);
    }
    uint16_t* const to = x + r * b.ld_x + c;  // rows end on a multiple of sixteen
    *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(to + b.x_term) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  });
}

// CTAs of a matrix: what fills the device, no more than there are rows for.
int grid_of(const MuonBatch& b, int sm_count) {
  int per = 8;
  while (per < kThreads && 8 * per < b.C) per <<= 1;
  const int high = kThreads / per, rows = (b.R + high - 1) / high, room = std::max(1, kCtas * sm_count / b.n);
  const int most = room < kMuonPartials ? room : kMuonPartials;
  return rows < most ? rows : most;
}

}  // namespace

cudaError_t launch_muon_moments(const MuonBatch& b, int sm_count, cudaStream_t s) {
  return launch_pdl(b.step ? muon_moments_kernel<true> : muon_moments_kernel<false>, dim3(grid_of(b, sm_count), b.n), dim3(kThreads), 0, s, b);
}
cudaError_t launch_muon_scale(const MuonBatch& b, int sm_count, cudaStream_t s) {
  const int grid = grid_of(b, sm_count);
  return launch_pdl(b.step ? muon_scale_kernel<true> : muon_scale_kernel<false>, dim3(grid, b.n), dim3(kThreads), 0, s, b, grid);
}

}  // namespace sffn
