// The optimiser's kernels: one launch goes over a whole list of tensors, whose addresses and sizes travel in the
// kernel's parameters (nothing is copied to the device first, and a captured launch replays).
//
//   grad_norm_kernel     sqrt(sum g^2): every CTA leaves one partial sum in 64 bits, the last one to finish adds them up
//   adamw_kernel         the step itself; a warp owns 256 consecutive entries, which is also a group of 8-bit moments
//   adamw_values_kernel  8-bit moments as the fp32 values they stand for
//
// All three are bound by the bytes they move.
#include "optim_kernels.cuh"

#include <math.h>

#include "common.cuh"

namespace sffn {
namespace {

constexpr int kGroup = 256;   // entries of a warp's piece, and of a group of 8-bit moments
constexpr int kPer = kGroup / 32;
constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: a group whose largest value is below is stored as zeros

// Which tensor a piece belongs to: pieces are numbered through the list, and a warp meets them in ascending order.
template <typename List>
__device__ __forceinline__ void advance(const List& list, uint32_t piece, int& e) {
  while (e + 1 < list.n && piece >= list.e[e + 1].begin) ++e;
}

// ---- norm ------------------------------------------------------------------------------------------------------------

constexpr int kNormThreads = 512;
constexpr int kNormLoads = 4;                         // 16-byte loads of a lane in flight
constexpr int kNormPiece = 32 * 16 * kNormLoads;      // bytes of a warp's piece
constexpr int kNormMaxGrid = 1024;
static_assert(256 + 8 * kNormMaxGrid + 16 <= SFFN_GRAD_NORM_WORKSPACE, "partial sums fit");

struct NormEntry {
  const void* data;
  long long n;
  uint32_t begin;  // number of its first piece
  uint32_t dtype;
};
template <int N>
struct NormList {
  int n, first, last;  // first / last launch of a call
  uint32_t pieces;
  float* norm;
  uint32_t* counter;   // CTAs that have left their partial sum; 0 between calls
  double* partial;     // [grid], then the sum of the call's earlier launches
  NormEntry e[N];
};

__device__ __forceinline__ float sum_squares(const uint4& v, bool bf16, float acc) {
  if (bf16) {
    float f[8];
    Elem<__nv_bfloat16>::unpack(v, f);
    float2 a = make_float2(acc, 0.f);
#pragma unroll
    for (int i = 0; i < 8; i += 2) a = fma2(make_float2(f[i], f[i + 1]), make_float2(f[i], f[i + 1]), a);
    return a.x + a.y;
  }
  float f[4];
  Elem<float>::unpack(v, f);
  float2 a = make_float2(acc, 0.f);
  a = fma2(make_float2(f[0], f[1]), make_float2(f[0], f[1]), a);
  a = fma2(make_float2(f[2], f[3]), make_float2(f[2], f[3]), a);
  return a.x + a.y;
}

template <int N>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormList<N> list) {
  __shared__ double warp_total[kNormThreads / 32];
  __shared__ bool last_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t warps = gridDim.x * (kNormThreads / 32);
  float acc[kNormLoads] = {};
  double total = 0.0;
  int e = 0, since = 0;
  for (uint32_t piece = blockIdx.x * (kNormThreads / 32) + warp; piece < list.pieces; piece += warps) {
    advance(list, piece, e);
    const NormEntry& t = list.e[e];
    const bool bf16 = t.dtype == SFFN_BF16;
    const int esz = bf16 ? 2 : 4;
    const long long first = (long long)(piece - t.begin) * (kNormPiece / esz);
    const char* p = static_cast<const char*>(t.data) + first * esz;
    const long long left = t.n - first;
    if (left >= kNormPiece / esz && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
      uint4 v[kNormLoads];
#pragma unroll
      for (int i = 0; i < kNormLoads; ++i) v[i] = ld_stream16(p + (i * 32 + lane) * 16);
#pragma unroll
      for (int i = 0; i < kNormLoads; ++i) acc[i] = sum_squares(v[i], bf16, acc[i]);
    } else {  // a tensor's end, or one that does not start on 16 bytes
      const int count = (int)(left < kNormPiece / esz ? left : kNormPiece / esz);
      for (int i = lane; i < count; i += 32) {
        const float g = bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]) : reinterpret_cast<const float*>(p)[i];
        acc[0] = fmaf(g, g, acc[0]);
      }
    }
    if (++since == 32) {  // short runs in 32 bits, their sums in 64
#pragma unroll
      for (int i = 0; i < kNormLoads; ++i) { total += (double)acc[i]; acc[i] = 0.f; }
      since = 0;
    }
  }
#pragma unroll
  for (int i = 0; i < kNormLoads; ++i) total += (double)acc[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) warp_total[warp] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    double sum = 0.0;
    for (int w = 0; w < kNormThreads / 32; ++w) sum += warp_total[w];
    list.partial[blockIdx.x] = sum;
    __threadfence();
    last_cta = atomicAdd(list.counter, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last_cta) return;
  // All partial sums are there: they are added in an order that does not depend on which CTA does it.
  double sum = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kNormThreads) sum += __ldcg(list.partial + i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) warp_total[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = list.first ? 0.0 : __ldcg(list.partial + kNormMaxGrid);
    for (int w = 0; w < kNormThreads / 32; ++w) sum += warp_total[w];
    list.partial[kNormMaxGrid] = sum;
    if (list.last) *list.norm = (float)sqrt(sum);
    *list.counter = 0;
  }
}

template <int N>
cudaError_t norm_launches(const sffn_tensor* t, int n, float* norm, void* workspace, int sm_count, cudaStream_t s) {
  int at = 0;
  bool first = true;
  do {
    NormList<N> list;
    list.n = 0;
    long long pieces = 0;
    for (; at < n && list.n < N; ++at) {
      if (t[at].n == 0) continue;
      const long long per = kNormPiece / (t[at].dtype == SFFN_BF16 ? 2 : 4);
      const long long own = (t[at].n + per - 1) / per;
      if (pieces + own > 0xffffffffll - (1 << 20)) break;
      NormEntry& e = list.e[list.n++];
      e.data = t[at].data;
      e.n = t[at].n;
      e.begin = (uint32_t)pieces;
      e.dtype = (uint32_t)t[at].dtype;
      pieces += own;
    }
    list.first = first;
    list.last = at >= n;
    list.pieces = (uint32_t)pieces;
    list.norm = norm;
    list.counter = static_cast<uint32_t*>(workspace);
    list.partial = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
    const long long want = (pieces + kNormThreads / 32 - 1) / (kNormThreads / 32);
    int grid = 4 * sm_count < kNormMaxGrid ? 4 * sm_count : kNormMaxGrid;
    if (want < grid) grid = want > 0 ? (int)want : 1;
    grad_norm_kernel<N><<<grid, kNormThreads, 0, s>>>(list);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    first = false;
  } while (at < n);
  return cudaSuccess;
}

// ---- AdamW -----------------------------------------------------------------------------------------------------------

constexpr int kStepThreads = 256;

// What a tensor's kinds of storage are, in one word.
constexpr uint32_t kPBf16 = 1, kGBf16 = 2, kMaster = 4, kCodes = 8, kWide = 16;  // kWide: every pointer allows vector accesses

struct StepEntry {
  void* p;
  const void* g;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  long long n;
  uint32_t begin, kind;
  float decay, rate;  // 1 - lr weight_decay, lr / (1 - beta1^step)
};
template <int N>
struct StepList {
  int n;
  uint32_t pieces;
  const float* grad_norm;
  float max_norm, beta1, one_beta1, beta2, one_beta2, root_bc2, eps;  // root_bc2: 1 / sqrt(1 - beta2^step)
  StepEntry e[N];
};

__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The number of edges (k + 1/2)^2, k < 127, at or below q: a square root that may be off by its last bits, then the edges
// themselves (exact in 32 bits) decide.
__device__ __forceinline__ int code_of_square(float q) {
  float c = fminf(floorf(sqrt_approx(q) + 0.5f), 127.f);
  const float up = fmaf(c, c, c) + 0.25f, down = fmaf(c, c, -c) + 0.25f;  // c <= 127: exact
  if (q >= up) c += 1.f;
  else if (q < down) c -= 1.f;
  return (int)fminf(fmaxf(c, 0.f), 127.f);
}
// The same with edges (k + 1/2)^4, k < 255, each the rounded square of an exact (k + 1/2)^2.
__device__ __forceinline__ int code_of_fourth(float q) {
  float c = fminf(floorf(sqrt_approx(sqrt_approx(q)) + 0.5f), 255.f);
  float up = fmaf(c, c, c) + 0.25f, down = fmaf(c, c, -c) + 0.25f;
  up = __fmul_rn(up, up);
  down = __fmul_rn(down, down);
  if (q >= up) c += 1.f;
  else if (q < down) c -= 1.f;
  return (int)fminf(fmaxf(c, 0.f), 255.f);
}

__device__ __forceinline__ float code_m(int c, float unit) { return __fmul_rn((float)(c * abs(c)), unit); }
__device__ __forceinline__ float code_v(int c, float unit) {
  const float t = (float)(c * c);
  return __fmul_rn(__fmul_rn(t, t), unit);
}
__device__ __forceinline__ float unit_m(float scale) { return __fmul_rn(scale, (float)(1.0 / (127.0 * 127.0))); }
__device__ __forceinline__ float unit_v(float scale) { return __fmul_rn(scale, (float)(1.0 / (255.0 * 255.0 * 255.0 * 255.0))); }

// A group's scale as it is stored and what its values are multiplied by first: 0 for a group of zeros (or one below
// kTiny), and for a group that holds an infinity or a NaN, whose scale then says so for all of it.
__device__ __forceinline__ float group_scale(float most, float& inverse) {
  const bool fine = most >= kTiny && most <= 3.402823466e38f;
  inverse = fine ? __frcp_rn(most) : 0.f;
  return fine || !(most < kTiny) ? most : 0.f;
}
__device__ __forceinline__ float warp_most(float mine) {  // values >= 0 order like their bits, NaN above all
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mine) & 0x7fffffffu));
}

__device__ __forceinline__ void load8_f32(const float* p, uint4* raw) {
  raw[0] = *reinterpret_cast<const uint4*>(p);
  raw[1] = *reinterpret_cast<const uint4*>(p + 4);
}
__device__ __forceinline__ void floats_of(const uint4* raw, bool bf16, float* f) {
  if (bf16) {
    Elem<__nv_bfloat16>::unpack(raw[0], f);
  } else {
    Elem<float>::unpack(raw[0], f);
    Elem<float>::unpack(raw[1], f + 4);
  }
}
__device__ __forceinline__ void store8_f32(float* p, const float* f) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// One step of one entry; the products and sums of the moments are rounded one by one, so that codes do not depend on
// how an expression is contracted.
template <typename List>
__device__ __forceinline__ void step_entry(const List& c, const StepEntry& t, float coef, float g, float& w, float& m, float& v) {
  g = __fmul_rn(g, coef);
  m = __fadd_rn(__fmul_rn(m, c.beta1), __fmul_rn(g, c.one_beta1));
  v = __fadd_rn(__fmul_rn(v, c.beta2), __fmul_rn(__fmul_rn(g, g), c.one_beta2));
  const float denominator = fmaf(sqrt_approx(v), c.root_bc2, c.eps);
  w = w * t.decay - __fdividef(m, denominator) * t.rate;
}

// Entry j of a lane: 8 lane + j where vectors are used, 32 j + lane otherwise.
template <int N>
__global__ void __launch_bounds__(kStepThreads) adamw_kernel(const __grid_constant__ StepList<N> list) {
  const int lane = threadIdx.x & 31;
  const uint32_t warps = gridDim.x * (kStepThreads / 32);
  float coef = 1.f;
  if (list.grad_norm) {
    const float norm = *list.grad_norm;
    if (!(fabsf(norm) <= 3.402823466e38f)) return;  // the step is left out
    coef = fminf(__fdiv_rn(list.max_norm, __fadd_rn(norm, 1e-6f)), 1.f);
  }
  int e = 0;
  for (uint32_t piece = blockIdx.x * (kStepThreads / 32) + (threadIdx.x >> 5); piece < list.pieces; piece += warps) {
    advance(list, piece, e);
    const StepEntry& t = list.e[e];
    const uint32_t kind = t.kind, group = piece - t.begin;
    const long long first = (long long)group * kGroup;
    const bool codes = kind & kCodes, p_bf16 = kind & kPBf16, g_bf16 = kind & kGBf16, master = kind & kMaster;
    const bool wide = (kind & kWide) && t.n - first >= kGroup;
    const int left = (int)min((long long)kGroup, t.n - first);
    float w[kPer], g[kPer], m[kPer], v[kPer], sm = 0.f, sv = 0.f;
    if (codes) {
      sm = t.m_scale[group];
      sv = t.v_scale[group];
    }
    if (wide) {
      const long long at = first + lane * kPer;
      uint4 rw[2], rg[2], rm[2], rv[2];
      // every load is under way before the first value is looked at
      if (master) load8_f32(t.master + at, rw);
      else if (p_bf16) rw[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.p) + at);
      else load8_f32(static_cast<const float*>(t.p) + at, rw);
      if (g_bf16) rg[0] = ld_stream16(static_cast<const __nv_bfloat16*>(t.g) + at);
      else {
        rg[0] = ld_stream16(static_cast<const float*>(t.g) + at);
        rg[1] = ld_stream16(static_cast<const float*>(t.g) + at + 4);
      }
      if (codes) {
        const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(t.m) + at);
        const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at);
        rm[0] = make_uint4(a.x, a.y, 0, 0);
        rv[0] = make_uint4(b.x, b.y, 0, 0);
      } else {
        load8_f32(static_cast<const float*>(t.m) + at, rm);
        load8_f32(static_cast<const float*>(t.v) + at, rv);
      }
      floats_of(rw, p_bf16 && !master, w);
      floats_of(rg, g_bf16, g);
      if (codes) {
        const float um = unit_m(sm), uv = unit_v(sv);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          m[j] = code_m((int)(int8_t)((j < 4 ? rm[0].x : rm[0].y) >> (8 * (j & 3))), um);
          v[j] = code_v((int)(uint8_t)((j < 4 ? rv[0].x : rv[0].y) >> (8 * (j & 3))), uv);
        }
      } else {
        floats_of(rm, false, m);
        floats_of(rv, false, v);
      }
    } else {
      const float um = unit_m(sm), uv = unit_v(sv);
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        w[j] = g[j] = m[j] = v[j] = 0.f;
        const int i = 32 * j + lane;
        if (i >= left) continue;
        const long long at = first + i;
        w[j] = master ? t.master[at] : p_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.p)[at]) : static_cast<const float*>(t.p)[at];
        g[j] = g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.g)[at]) : static_cast<const float*>(t.g)[at];
        m[j] = codes ? code_m(static_cast<const int8_t*>(t.m)[at], um) : static_cast<const float*>(t.m)[at];
        v[j] = codes ? code_v(static_cast<const uint8_t*>(t.v)[at], uv) : static_cast<const float*>(t.v)[at];
      }
    }
    float most_m = 0.f, most_v = 0.f;
    uint32_t bits_m = 0, bits_v = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      step_entry(list, t, coef, g[j], w[j], m[j], v[j]);
      if (!wide && 32 * j + lane >= left) m[j] = v[j] = 0.f;
      bits_m = max(bits_m, __float_as_uint(m[j]) & 0x7fffffffu);
      bits_v = max(bits_v, __float_as_uint(v[j]) & 0x7fffffffu);
    }
    int8_t cm[kPer];
    uint8_t cv[kPer];
    if (codes) {
      most_m = warp_most(__uint_as_float(bits_m));
      most_v = warp_most(__uint_as_float(bits_v));
      float im, iv;
      sm = group_scale(most_m, im);
      sv = group_scale(most_v, iv);
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int a = code_of_square(__fmul_rn(__fmul_rn(fabsf(m[j]), im), 16129.f));
        const int b = code_of_fourth(__fmul_rn(__fmul_rn(v[j], iv), 4228250624.f));
        cm[j] = (int8_t)(im == 0.f ? 0 : m[j] < 0.f ? -a : a);
        cv[j] = (uint8_t)(iv == 0.f ? 0 : v[j] > 0.f ? max(b, 1) : b);
      }
      if (lane == 0) {
        t.m_scale[group] = sm;
        t.v_scale[group] = sv;
      }
    }
    if (wide) {
      const long long at = first + lane * kPer;
      if (p_bf16) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(t.p) + at) =
            make_uint4(two_bf16(w[0], w[1]), two_bf16(w[2], w[3]), two_bf16(w[4], w[5]), two_bf16(w[6], w[7]));
        if (master) store8_f32(t.master + at, w);
      } else {
        store8_f32(static_cast<float*>(t.p) + at, w);
      }
      if (codes) {
        uint32_t a[2] = {0, 0}, b[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          a[j >> 2] |= (uint32_t)(uint8_t)cm[j] << (8 * (j & 3));
          b[j >> 2] |= (uint32_t)cv[j] << (8 * (j & 3));
        }
        *reinterpret_cast<uint2*>(static_cast<int8_t*>(t.m) + at) = make_uint2(a[0], a[1]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + at) = make_uint2(b[0], b[1]);
      } else {
        store8_f32(static_cast<float*>(t.m) + at, m);
        store8_f32(static_cast<float*>(t.v) + at, v);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int i = 32 * j + lane;
        if (i >= left) continue;
        const long long at = first + i;
        if (p_bf16) {
          static_cast<__nv_bfloat16*>(t.p)[at] = __float2bfloat16(w[j]);
          if (master) t.master[at] = w[j];
        } else {
          static_cast<float*>(t.p)[at] = w[j];
        }
        if (codes) {
          static_cast<int8_t*>(t.m)[at] = cm[j];
          static_cast<uint8_t*>(t.v)[at] = cv[j];
        } else {
          static_cast<float*>(t.m)[at] = m[j];
          static_cast<float*>(t.v)[at] = v[j];
        }
      }
    }
  }
}

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Launches a kernel over a list of tensors, at most N at a time: `fill` writes one tensor's entry.
template <int N, typename List, typename Kernel, typename Fill>
cudaError_t list_launches(List& list, Kernel kernel, int n, const sffn_adamw_tensor* t, int sm_count, cudaStream_t s, Fill fill) {
  for (int at = 0; at < n;) {
    list.n = 0;
    long long pieces = 0;
    for (; at < n && list.n < N; ++at) {
      const long long own = (t[at].n + kGroup - 1) / kGroup;
      if (own == 0) continue;
      if (pieces + own > 0xffffffffll - (1 << 20)) break;
      auto& e = list.e[list.n++];
      e.begin = (uint32_t)pieces;
      fill(e, at);
      pieces += own;
    }
    if (pieces == 0) continue;
    list.pieces = (uint32_t)pieces;
    int per_sm = 0;
    cudaError_t err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kStepThreads, 0);
    if (err != cudaSuccess) return err;
    const long long want = (pieces + kStepThreads / 32 - 1) / (kStepThreads / 32);
    const long long room = (long long)(per_sm > 0 ? per_sm : 1) * sm_count;
    kernel<<<(unsigned)(want < room ? want : room), kStepThreads, 0, s>>>(list);
    err = cudaGetLastError();
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

template <int N>
cudaError_t adamw_launches(const sffn_adamw_tensor* t, int n, const sffn_adamw_config& c, int sm_count, cudaStream_t s) {
  StepList<N> list;
  list.grad_norm = c.grad_norm;
  list.max_norm = (float)c.max_norm;
  list.beta1 = (float)c.beta1;
  list.one_beta1 = (float)(1.0 - c.beta1);
  list.beta2 = (float)c.beta2;
  list.one_beta2 = (float)(1.0 - c.beta2);
  list.eps = (float)c.eps;
  const double bc1 = 1.0 - pow(c.beta1, (double)c.step), bc2 = 1.0 - pow(c.beta2, (double)c.step);
  list.root_bc2 = (float)(1.0 / sqrt(bc2));
  return list_launches<N>(list, adamw_kernel<N>, n, t, sm_count, s, [&](StepEntry& e, int i) {
    const sffn_adamw_tensor& a = t[i];
    e.p = a.p; e.g = a.g; e.master = a.master; e.m = a.m; e.v = a.v; e.m_scale = a.m_scale; e.v_scale = a.v_scale; e.n = a.n;
    e.kind = (a.p_dtype == SFFN_BF16 ? kPBf16 : 0) | (a.g_dtype == SFFN_BF16 ? kGBf16 : 0) | (a.master ? kMaster : 0) | (a.state_bits == 8 ? kCodes : 0);
    const uintptr_t sa = a.state_bits == 8 ? 8 : 16;
    if (aligned_to(a.p, 16) && aligned_to(a.g, 16) && aligned_to(a.master, 16) && aligned_to(a.m, sa) && aligned_to(a.v, sa)) e.kind |= kWide;
    e.decay = (float)(1.0 - a.lr * a.weight_decay);
    e.rate = (float)(a.lr / bc1);
  });
}

// ---- values of 8-bit moments -----------------------------------------------------------------------------------------

struct ValueEntry {
  const int8_t* m;
  const uint8_t* v;
  const float *m_scale, *v_scale;
  float *m_out, *v_out;
  long long n;
  uint32_t begin, wide;
};
template <int N>
struct ValueList {
  int n;
  uint32_t pieces;
  ValueEntry e[N];
};

template <int N>
__global__ void __launch_bounds__(kStepThreads) adamw_values_kernel(const __grid_constant__ ValueList<N> list) {
  const int lane = threadIdx.x & 31;
  const uint32_t warps = gridDim.x * (kStepThreads / 32);
  int e = 0;
  for (uint32_t piece = blockIdx.x * (kStepThreads / 32) + (threadIdx.x >> 5); piece < list.pieces; piece += warps) {
    advance(list, piece, e);
    const ValueEntry& t = list.e[e];
    const uint32_t group = piece - t.begin;
    const long long first = (long long)group * kGroup;
    const int left = (int)min((long long)kGroup, t.n - first);
    const float um = t.m_out ? unit_m(t.m_scale[group]) : 0.f, uv = t.v_out ? unit_v(t.v_scale[group]) : 0.f;
    if (t.wide && left == kGroup) {  // four entries of a lane in each half, so that a warp's stores are 512 bytes in a row
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const long long at = first + 128 * h + 4 * lane;
        if (t.m_out) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(t.m + at);
          *reinterpret_cast<float4*>(t.m_out + at) = make_float4(code_m((int8_t)w, um), code_m((int8_t)(w >> 8), um),
                                                                 code_m((int8_t)(w >> 16), um), code_m((int8_t)(w >> 24), um));
        }
        if (t.v_out) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(t.v + at);
          *reinterpret_cast<float4*>(t.v_out + at) = make_float4(code_v((uint8_t)w, uv), code_v((uint8_t)(w >> 8), uv),
                                                                 code_v((uint8_t)(w >> 16), uv), code_v((uint8_t)(w >> 24), uv));
        }
      }
    } else {
      for (int i = lane; i < left; i += 32) {
        if (t.m_out) t.m_out[first + i] = code_m(t.m[first + i], um);
        if (t.v_out) t.v_out[first + i] = code_v(t.v[first + i], uv);
      }
    }
  }
}

template <int N>
cudaError_t value_launches(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, int sm_count, cudaStream_t s) {
  ValueList<N> list;
  return list_launches<N>(list, adamw_values_kernel<N>, n, t, sm_count, s, [&](ValueEntry& e, int i) {
    e.m = static_cast<const int8_t*>(t[i].m);
    e.v = static_cast<const uint8_t*>(t[i].v);
    e.m_scale = t[i].m_scale;
    e.v_scale = t[i].v_scale;
    e.m_out = m_out ? m_out[i] : nullptr;
    e.v_out = v_out ? v_out[i] : nullptr;
    e.n = t[i].n;
    e.wide = aligned_to(e.m, 4) && aligned_to(e.v, 4) && aligned_to(e.m_out, 16) && aligned_to(e.v_out, 16);
  });
}

// A launch carries its list in the kernel's parameters (at most 32764 bytes).  Short lists take a small one: the
// parameters are copied at every launch.
constexpr int kShort = 40;
constexpr int kLongNorm = 1300, kLongStep = 360;
static_assert(sizeof(NormList<kLongNorm>) <= 32764 && sizeof(StepList<kLongStep>) <= 32764 && sizeof(ValueList<kLongStep>) <= 32764, "kernel parameters");

}  // namespace

cudaError_t launch_grad_norm(const sffn_tensor* t, int n, float* norm, void* workspace, int sm_count, cudaStream_t s) {
  return n <= kShort ? norm_launches<kShort>(t, n, norm, workspace, sm_count, s) : norm_launches<kLongNorm>(t, n, norm, workspace, sm_count, s);
}

cudaError_t launch_adamw(const sffn_adamw_tensor* t, int n, const sffn_adamw_config& c, int sm_count, cudaStream_t s) {
  return n <= kShort ? adamw_launches<kShort>(t, n, c, sm_count, s) : adamw_launches<kLongStep>(t, n, c, sm_count, s);
}

cudaError_t launch_adamw_values(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, int sm_count, cudaStream_t s) {
  return n <= kShort ? value_launches<kShort>(t, n, m_out, v_out, sm_count, s) : value_launches<kLongStep>(t, n, m_out, v_out, sm_count, s);
}

}  // namespace sffn
