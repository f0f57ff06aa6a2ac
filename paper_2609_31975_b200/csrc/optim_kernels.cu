// The optimiser's kernels: one launch goes over a whole list of tensors, whose addresses and sizes travel in the
// kernel's parameters (nothing is copied to the device first, and a captured launch replays).
//
//   grad_norm_kernel     sqrt(sum g^2): every CTA leaves one partial sum in 64 bits, the last one to finish adds them up
//   adamw_kernel         the step itself; a warp owns 256 consecutive entries, which is also a group of 8-bit moments
//   adamw_values_kernel  8-bit moments as the fp32 values they stand for
//
// Bound by the bytes they move, the step with 8-bit moments also by its instructions (about 55 an entry, half of them on the ALU).
// B200, copies at 6.45 TB/s, calls in a loop: norm of 704 M bf16 entries 202 us (7.0 TB/s); step of 164 M entries with fp32 moments and
// copies 758 us (6.1 TB/s), of 64 tensors of 12.6 M entries in all 60 us (5.9 TB/s; 59 where the next launch may start under its tail); 235 M
// bf16 entries in 8 bits 489 us (4.8 TB/s), their values 405 us (5.8 TB/s).
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
constexpr int kNormLoads = 4;                         // 32-byte loads of a lane in flight
constexpr int kNormPiece = 32 * 32 * kNormLoads;      // bytes of a warp's piece
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

__device__ __forceinline__ float sum_squares(const uint32_t* w, bool bf16, float acc) {
  float2 a = make_float2(acc, 0.f), b = make_float2(0.f, 0.f);
  if (bf16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
      if (i & 1) b = fma2(f, f, b);
      else a = fma2(f, f, a);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      if (i & 1) b = fma2(f, f, b);
      else a = fma2(f, f, a);
    }
  }
  return (a.x + a.y) + (b.x + b.y);
}
__device__ __forceinline__ void ld32(const void* p, uint32_t* w) {  // 32 bytes
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}

template <int N>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormList<N> list) {
  __shared__ double warp_total[kNormThreads / 32];
  __shared__ bool last_cta;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t warps = gridDim.x * (kNormThreads / 32);
  pdl_launch_dependents();
  pdl_wait();
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
    if (left >= kNormPiece / esz && (reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
      uint32_t v[kNormLoads][8];
#pragma unroll
      for (int i = 0; i < kNormLoads; ++i) ld32(p + (i * 32 + lane) * 32, v[i]);
#pragma unroll
      for (int i = 0; i < kNormLoads; ++i) acc[i] = sum_squares(v[i], bf16, acc[i]);
    } else {  // a tensor's end, or one that does not start on 32 bytes
      const int count = (int)(left < kNormPiece / esz ? left : kNormPiece / esz);
      for (int i = lane; i < count; i += 32) {
        const float g = bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]) : reinterpret_cast<const float*>(p)[i];
        acc[0] = fmaf(g, g, acc[0]);
      }
    }
    if (++since == 16) {  // short runs in 32 bits, their sums in 64
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
    const cudaError_t e = launch_pdl(grad_norm_kernel<N>, dim3(grid), dim3(kNormThreads), 0, s, list);
    if (e != cudaSuccess) return e;
    first = false;
  } while (at < n);
  return cudaSuccess;
}

// ---- AdamW -----------------------------------------------------------------------------------------------------------

constexpr int kStepThreads = 128;

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
  uint32_t pieces, run;  // run: groups of a piece
  const float* grad_norm;
  float max_norm, beta1, one_beta1, beta2, one_beta2, root_bc2, eps;  // root_bc2: 1 / sqrt(1 - beta2^step)
  StepEntry e[N];
};

// Pairs of fp32 in one register pair, each half as in the scalar operation -- but the compiler may fuse a product and the sum it
// goes into, which it does not do across halves taken apart (add_apart).
typedef unsigned long long f2;
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ void halves(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ float low(f2 v) { float a, b; halves(v, a, b); return a; }
__device__ __forceinline__ float high(f2 v) { float a, b; halves(v, a, b); return b; }

__device__ __forceinline__ f2 add_apart(f2 a, f2 b) { return pack2(__fadd_rn(low(a), low(b)), __fadd_rn(high(a), high(b))); }

__device__ __forceinline__ float sqrt_approx(float x) {  // what is below 2^-126 counts as zero
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

constexpr float kMagic = 12582912.f;   // 1.5 2^23: a small number added to it is rounded to an integer, in its low bits

// Codes: the number of edges (k + 1/2)^2, k < 127 (for v: the rounded squares of those, k < 255) at or below q.  An approximate root
// rounded to an integer is the code unless it lies within kNear of an edge.  That leaves one group in fifteen, where the edges
// are asked: the root, made a little too small, is rounded to an integer c that the code is never below and at most one above, and
// whether q reaches the edge above c is seen in numbers that fp32 holds exactly.
// (Roots are off by at most 255 (5e-7 / 2 + 2e-7) = 1.2e-4: products and approximate roots of 2 to 5 roundings.)
constexpr float kNear = 1.5e-4f, kMargin = 2e-4f;

__device__ __forceinline__ uint32_t code_of_square(float m, float q) {
  const float n = sqrt_approx(q) - kMargin + kMagic, c = n - kMagic;
  int code = __float_as_int(n) - __float_as_int(kMagic);
  if (fmaf(-c, c, q) >= c + 0.25f) ++code;
  return m < 0.f ? -code : code;
}
__device__ __forceinline__ uint32_t code_of_fourth(float v, float q) {
  const float n = sqrt_approx(sqrt_approx(q)) - kMargin + kMagic, c = n - kMagic;
  const float t = fmaf(c, c, c + 0.25f);  // (c + 1/2)^2, exact
  int code = __float_as_int(n) - __float_as_int(kMagic);
  if (q >= __fmul_rn(t, t)) ++code;
  return max(code, v > 0.f ? 1 : 0);      // what is not zero stays so: it divides
}

// Low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// The codes of eight entries by the edges: m's in x, y, v's in z, w.  Out of line: few groups come here, and its registers would be
// the others'.
__device__ __noinline__ uint4 exact_codes(f2 m0, f2 m1, f2 m2, f2 m3, f2 v0, f2 v1, f2 v2, f2 v3, float im, float iv) {
  const f2 m[4] = {m0, m1, m2, m3}, v[4] = {v0, v1, v2, v3};
  uint32_t a[8], b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float mj = j & 1 ? high(m[j / 2]) : low(m[j / 2]), vj = j & 1 ? high(v[j / 2]) : low(v[j / 2]);
    a[j] = code_of_square(mj, __fmul_rn(__fmul_rn(fabsf(mj), im), 16129.f));
    b[j] = code_of_fourth(vj, __fmul_rn(__fmul_rn(vj, iv), 4228250624.f));
  }
  return make_uint4(low_bytes(a[0], a[1], a[2], a[3]), low_bytes(a[4], a[5], a[6], a[7]), low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
}

__device__ __forceinline__ float code_m(int c, float unit) { return __fmul_rn((float)(c * abs(c)), unit); }
__device__ __forceinline__ float code_v(int c, float unit) {
  const float t = (float)(c * c);
  return __fmul_rn(__fmul_rn(t, t), unit);
}
// Four codes of a word, without integer conversions: the byte (m: + 128) goes under the exponent of 2^23.
__device__ __forceinline__ void codes_m(uint32_t w, f2 unit, f2* v) {
  w ^= 0x80808080u;
  const f2 bias = both(-8388736.f);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f2 c = add2_b64(pack2(__uint_as_float(__byte_perm(w, 0x4b000000u, i ? 0x7442 : 0x7440)), __uint_as_float(__byte_perm(w, 0x4b000000u, i ? 0x7443 : 0x7441))), bias);
    v[i] = mul2(pack2(__fmul_rn(low(c), fabsf(low(c))), __fmul_rn(high(c), fabsf(high(c)))), unit);
  }
}
__device__ __forceinline__ void codes_v(uint32_t w, f2 unit, f2* v) {
  const f2 bias = both(-8388608.f);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f2 c = add2_b64(pack2(__uint_as_float(__byte_perm(w, 0x4b000000u, i ? 0x7442 : 0x7440)), __uint_as_float(__byte_perm(w, 0x4b000000u, i ? 0x7443 : 0x7441))), bias);
    const f2 t = mul2(c, c);
    v[i] = mul2(mul2(t, t), unit);
  }
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

__device__ __forceinline__ void st32(void* p, const f2* v) {
  asm volatile("st.global.v4.b64 [%0], {%1,%2,%3,%4};" ::"l"(p), "l"(v[0]), "l"(v[1]), "l"(v[2]), "l"(v[3]) : "memory");
}
__device__ __forceinline__ void ld16(const void* p, uint32_t* w) {
  asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
}
__device__ __forceinline__ void pairs_of(const uint32_t* w, bool bf16, f2* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f[i] = bf16 ? pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)) : pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}
__device__ __forceinline__ uint32_t two_bf16(f2 v) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(low(v), high(v));
  return *reinterpret_cast<const uint32_t*>(&b);
}

// Eight entries of a lane as four pairs.  Entry j of a lane: 8 lane + j where vectors are used (WIDE), 32 j + lane otherwise.
// CODES: the moments are held in codes.  HALF: bf16 parameters without copies, which the kernel then need not look up.  FULL: roots and
// quotients over all of fp32 (see fast_roots).
template <bool CODES, bool WIDE, bool HALF, bool FULL, typename List>
__device__ __forceinline__ void finish_group(const List& c, const StepEntry& t, uint32_t group, float coef, int lane, f2* w, f2* g, f2* m, f2* v) {
  const uint32_t kind = t.kind;
  const long long first = (long long)group * kGroup;
  const bool p_bf16 = HALF || (kind & kPBf16), master = !HALF && (kind & kMaster);
  const int left = WIDE ? kGroup : (int)min((long long)kGroup, t.n - first);
  float sm, sv;
  float most_m = 0.f, most_v = 0.f;
  f2 root[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    // products and sums of the moments are rounded one by one: codes do not depend on how an expression is contracted
    g[q] = mul2(g[q], both(coef));
    m[q] = add_apart(mul2(m[q], both(c.beta1)), mul2(g[q], both(c.one_beta1)));
    v[q] = add_apart(mul2(v[q], both(c.beta2)), mul2(mul2(g[q], g[q]), both(c.one_beta2)));
    root[q] = FULL ? pack2(__fsqrt_rn(low(v[q])), __fsqrt_rn(high(v[q]))) : pack2(sqrt_approx(low(v[q])), sqrt_approx(high(v[q])));
    const f2 below = fma2_b64(root[q], both(c.root_bc2), both(c.eps));
    const f2 part = FULL ? pack2(__fdiv_rn(low(m[q]), low(below)), __fdiv_rn(high(m[q]), high(below)))
                         : mul2(m[q], pack2(rcp_approx(low(below)), rcp_approx(high(below))));
    w[q] = fma2_b64(part, both(-t.rate), mul2(w[q], both(t.decay)));
    if (CODES) {  // entries past the end are zeros, of weight zero
      most_m = max_nan(most_m, max_nan(fabsf(low(m[q])), fabsf(high(m[q]))));
      most_v = max_nan(most_v, max_nan(low(v[q]), high(v[q])));
    }
  }
  uint4 codes = make_uint4(0, 0, 0, 0);  // m's in x, y, v's in z, w
  if constexpr (CODES) {
    float im, iv;
    sm = group_scale(warp_most(most_m), im);
    sv = group_scale(warp_most(most_v), iv);
    const float half = 65025.f * sqrt_approx(iv);  // sqrt(255^4 / scale)
    float near = 0.f, least = 1.f;
    uint32_t a[8], b[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float m0, m1;
      halves(m[q], m0, m1);
      const f2 square = mul2(pack2(__fmul_rn(fabsf(m0), im), __fmul_rn(fabsf(m1), im)), both(16129.f));
      const f2 hr = mul2(root[q], both(half));
      const f2 sa = pack2(copysignf(sqrt_approx(low(square)), m0), copysignf(sqrt_approx(high(square)), m1));
      const f2 sb = pack2(sqrt_approx(low(hr)), sqrt_approx(high(hr)));
      const f2 na = add2_b64(sa, both(kMagic)), nb = add2_b64(sb, both(kMagic));
      const f2 da = fma2_b64(add2_b64(na, both(-kMagic)), both(-1.f), sa), db = fma2_b64(add2_b64(nb, both(-kMagic)), both(-1.f), sb);
      near = fmaxf(near, fmaxf(fabsf(low(da)), fabsf(high(da))));
      near = fmaxf(near, fmaxf(fabsf(low(db)), fabsf(high(db))));
      least = fminf(least, fminf(low(sb), high(sb)));
      a[2 * q] = __float_as_uint(low(na)); a[2 * q + 1] = __float_as_uint(high(na));
      b[2 * q] = __float_as_uint(low(nb)); b[2 * q + 1] = __float_as_uint(high(nb));
    }
    codes = make_uint4(low_bytes(a[0], a[1], a[2], a[3]), low_bytes(a[4], a[5], a[6], a[7]), low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
    // The edges decide: a root near one; a v whose code would be 0, as 0 is for zeros only (a group of nothing else aside); a scale
    // below 2^-90, as single values may have counted as zeros when their roots were taken.
    if (__any_sync(0xffffffffu, near > 0.5f - kNear || (least < 0.6f && iv != 0.f)) || iv > 1.2379400392853803e27f)
      codes = exact_codes(m[0], m[1], m[2], m[3], v[0], v[1], v[2], v[3], im, iv);
    if (im == 0.f) codes.x = codes.y = 0;
    if (iv == 0.f) codes.z = codes.w = 0;
    if (lane == 0) {
      t.m_scale[group] = sm;
      t.v_scale[group] = sv;
    }
  }
  if constexpr (WIDE) {
    const long long at = first + lane * kPer;
    if (p_bf16) {
      *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(t.p) + at) = make_uint4(two_bf16(w[0]), two_bf16(w[1]), two_bf16(w[2]), two_bf16(w[3]));
      if (master) st32(t.master + at, w);
    } else {
      st32(static_cast<float*>(t.p) + at, w);
    }
    if constexpr (CODES) {
      *reinterpret_cast<uint2*>(static_cast<int8_t*>(t.m) + at) = make_uint2(codes.x, codes.y);
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + at) = make_uint2(codes.z, codes.w);
    } else {
      st32(static_cast<float*>(t.m) + at, m);
      st32(static_cast<float*>(t.v) + at, v);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = 32 * j + lane;
      if (i >= left) continue;
      const long long at = first + i;
      const float wj = j & 1 ? high(w[j / 2]) : low(w[j / 2]);
      if (p_bf16) {
        static_cast<__nv_bfloat16*>(t.p)[at] = __float2bfloat16(wj);
        if (master) t.master[at] = wj;
      } else {
        static_cast<float*>(t.p)[at] = wj;
      }
      if (CODES) {
        static_cast<int8_t*>(t.m)[at] = (int8_t)((j < 4 ? codes.x : codes.y) >> (8 * (j & 3)));
        static_cast<uint8_t*>(t.v)[at] = (uint8_t)((j < 4 ? codes.z : codes.w) >> (8 * (j & 3)));
      } else {
        static_cast<float*>(t.m)[at] = j & 1 ? high(m[j / 2]) : low(m[j / 2]);
        static_cast<float*>(t.v)[at] = j & 1 ? high(v[j / 2]) : low(v[j / 2]);
      }
    }
  }
}

template <bool CODES, bool WIDE, bool FULL, typename List>
__device__ __forceinline__ void step_group(const List& c, const StepEntry& t, uint32_t group, float coef, int lane) {
  const uint32_t kind = t.kind;
  const long long first = (long long)group * kGroup;
  const bool p_bf16 = kind & kPBf16, g_bf16 = kind & kGBf16, master = kind & kMaster;
  const int left = WIDE ? kGroup : (int)min((long long)kGroup, t.n - first);
  f2 w[4], g[4], m[4], v[4];
  float sm = 0.f, sv = 0.f;
  if (CODES) {
    sm = t.m_scale[group];
    sv = t.v_scale[group];
  }
  if constexpr (WIDE) {
    const long long at = first + lane * kPer;
    uint32_t rw[8], rg[8], rm[8], rv[8];
    // every load is under way before the first value is looked at
    if (master) ld32(t.master + at, rw);
    else if (p_bf16) ld16(static_cast<const __nv_bfloat16*>(t.p) + at, rw);
    else ld32(static_cast<const float*>(t.p) + at, rw);
    if (g_bf16) ld16(static_cast<const __nv_bfloat16*>(t.g) + at, rg);
    else ld32(static_cast<const float*>(t.g) + at, rg);
    if constexpr (CODES) {
      const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(t.m) + at);
      const uint2 b = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at);
      rm[0] = a.x; rm[1] = a.y;
      rv[0] = b.x; rv[1] = b.y;
    } else {
      ld32(static_cast<const float*>(t.m) + at, rm);
      ld32(static_cast<const float*>(t.v) + at, rv);
    }
    pairs_of(rw, p_bf16 && !master, w);
    pairs_of(rg, g_bf16, g);
    if constexpr (CODES) {
      const f2 um = both(unit_m(sm)), uv = both(unit_v(sv));
      codes_m(rm[0], um, m); codes_m(rm[1], um, m + 2);
      codes_v(rv[0], uv, v); codes_v(rv[1], uv, v + 2);
    } else {
      pairs_of(rm, false, m);
      pairs_of(rv, false, v);
    }
  } else {
    const float um = unit_m(sm), uv = unit_v(sv);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float e[4][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = 32 * (2 * q + j) + lane;
        const long long at = first + i;
        e[0][j] = e[1][j] = e[2][j] = e[3][j] = 0.f;
        if (i >= left) continue;
        e[0][j] = master ? t.master[at] : p_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.p)[at]) : static_cast<const float*>(t.p)[at];
        e[1][j] = g_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(t.g)[at]) : static_cast<const float*>(t.g)[at];
        e[2][j] = CODES ? code_m(static_cast<const int8_t*>(t.m)[at], um) : static_cast<const float*>(t.m)[at];
        e[3][j] = CODES ? code_v(static_cast<const uint8_t*>(t.v)[at], uv) : static_cast<const float*>(t.v)[at];
      }
      w[q] = pack2(e[0][0], e[0][1]); g[q] = pack2(e[1][0], e[1][1]); m[q] = pack2(e[2][0], e[2][1]); v[q] = pack2(e[3][0], e[3][1]);
    }
  }
  finish_group<CODES, WIDE, false, FULL>(c, t, group, coef, lane, w, g, m, v);
}

// bf16 parameters and gradients, moments in codes: a group's 24 bytes a lane.
struct HalfGroup {
  uint4 w, g;
  uint2 m, v;
  float sm, sv;
  __device__ __forceinline__ void load(const StepEntry& t, uint32_t group, int lane) {
    const long long at = (long long)group * kGroup + lane * kPer;
    w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(t.p) + at);
    g = ld_stream16(static_cast<const __nv_bfloat16*>(t.g) + at);
    m = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(t.m) + at);
    v = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + at);
    sm = t.m_scale[group];
    sv = t.v_scale[group];
  }
  template <bool FULL, typename List>
  __device__ __forceinline__ void step(const List& c, const StepEntry& t, uint32_t group, float coef, int lane) const {
    f2 pw[4], pg[4], pm[4], pv[4];
    pairs_of(reinterpret_cast<const uint32_t*>(&w), true, pw);
    pairs_of(reinterpret_cast<const uint32_t*>(&g), true, pg);
    const f2 um = both(unit_m(sm)), uv = both(unit_v(sv));
    codes_m(m.x, um, pm); codes_m(m.y, um, pm + 2);
    codes_v(v.x, uv, pv); codes_v(v.y, uv, pv + 2);
    finish_group<true, true, true, FULL>(c, t, group, coef, lane, pw, pg, pm, pv);
  }
};

// What a launch's tensors have in common: moments in 32 bits; in codes; in codes, with bf16 parameters and gradients (and no copies).
enum { kWords = 0, kAnyCodes = 1, kHalfCodes = 2 };

// A warp's piece is `run` groups in a row.  The step of a group in codes is some 450 instructions a warp and its loads take as long:
// kHalfCodes has the next group's under way meanwhile (705 M entries: 2.14 -> 1.70 ms).  176 M entries: kHalfCodes 367 us (4.8 TB/s), kAnyCodes with
// copies 554 (5.1), of fp32 583 (4.9), of bf16 with fp32 gradients 541 (3.9).
template <int N, int WHAT, bool FULL>
__global__ void __launch_bounds__(kStepThreads, WHAT == kHalfCodes ? 5 : 6) adamw_kernel(const __grid_constant__ StepList<N> list) {
  const int lane = threadIdx.x & 31;
  const uint32_t warps = gridDim.x * (kStepThreads / 32);
  pdl_wait();  // and no launch_dependents: what follows may be an inference call, which reads weights before its own wait
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
    uint32_t group = (piece - t.begin) * list.run;
    const uint32_t end = min(group + list.run, (uint32_t)((t.n + kGroup - 1) / kGroup));
    const uint32_t wide_end = t.kind & kWide ? min(end, (uint32_t)(t.n / kGroup)) : group;
    if constexpr (WHAT == kHalfCodes) {
      HalfGroup now, next;
      if (group < wide_end) now.load(t, group, lane);
#pragma unroll 1
      for (; group < wide_end; ++group) {
        if (group + 1 < wide_end) next.load(t, group + 1, lane);
        now.template step<FULL>(list, t, group, coef, lane);
        now = next;
      }
    } else {
#pragma unroll 1
      for (; group < wide_end; ++group) step_group<WHAT != kWords, true, FULL>(list, t, group, coef, lane);
    }
#pragma unroll 1
    for (; group < end; ++group) step_group<WHAT != kWords, false, FULL>(list, t, group, coef, lane);
  }
}

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int what_of(const sffn_adamw_tensor& t) {
  return t.state_bits != 8 ? kWords : t.p_dtype == SFFN_BF16 && t.g_dtype == SFFN_BF16 && !t.master ? kHalfCodes : kAnyCodes;
}

// Launches a kernel over the tensors of a list that `mine` names, at most N at a time: `fill` writes one's entry.
template <int N, typename List, typename Kernel, typename Mine, typename Fill>
cudaError_t list_launches(List& list, Kernel kernel, int n, const sffn_adamw_tensor* t, int sm_count, cudaStream_t s, Mine mine, Fill fill) {
  for (int at = 0; at < n;) {
    list.n = 0;
    long long pieces = 0;
    for (; at < n && list.n < N; ++at) {
      const long long own = mine(t[at]) ? ((t[at].n + kGroup - 1) / kGroup + list.run - 1) / list.run : 0;
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
    err = launch_pdl(kernel, dim3((unsigned)(want < room ? want : room)), dim3(kStepThreads), 0, s, list);
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

// Groups of a piece: `most` once every warp of the device has several such pieces, one below, where pieces are what fills it.
inline uint32_t run_of(const sffn_adamw_tensor* t, int n, int sm_count, uint32_t most) {
  long long groups = 0;
  for (int i = 0; i < n; ++i) groups += (t[i].n + kGroup - 1) / kGroup;
  return groups > 256ll * most * sm_count ? most : 1;
}

// The fast root takes a v below 2^-126 for zero, which is up to 2^-63 / sqrt(1 - beta2^step) less to divide by: nothing, in fp32, beside an
// eps 2^25 times that, as all but the smallest are.
inline bool fast_roots(const sffn_adamw_config& c) { return c.eps * sqrt(1.0 - pow(c.beta2, (double)c.step)) >= 0x1p-38; }

template <int N, bool FULL>
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
  auto fill = [&](StepEntry& e, int i) {
    const sffn_adamw_tensor& a = t[i];
    e.p = a.p; e.g = a.g; e.master = a.master; e.m = a.m; e.v = a.v; e.m_scale = a.m_scale; e.v_scale = a.v_scale; e.n = a.n;
    e.kind = (a.p_dtype == SFFN_BF16 ? kPBf16 : 0) | (a.g_dtype == SFFN_BF16 ? kGBf16 : 0) | (a.master ? kMaster : 0) | (a.state_bits == 8 ? kCodes : 0);
    const uintptr_t state = a.state_bits == 8 ? 8 : 32;
    if (aligned_to(a.p, a.p_dtype == SFFN_BF16 ? 16 : 32) && aligned_to(a.g, a.g_dtype == SFFN_BF16 ? 16 : 32) && aligned_to(a.master, 32) &&
        aligned_to(a.m, state) && aligned_to(a.v, state))
      e.kind |= kWide;
    e.decay = (float)(1.0 - a.lr * a.weight_decay);
    e.rate = (float)(a.lr / bc1);
  };
  list.run = 1;
  cudaError_t err = list_launches<N>(list, adamw_kernel<N, kWords, FULL>, n, t, sm_count, s, [](const sffn_adamw_tensor& a) { return what_of(a) == kWords; }, fill);
  if (err != cudaSuccess) return err;
  list.run = run_of(t, n, sm_count, 16);
  err = list_launches<N>(list, adamw_kernel<N, kHalfCodes, FULL>, n, t, sm_count, s, [](const sffn_adamw_tensor& a) { return what_of(a) == kHalfCodes; }, fill);
  if (err != cudaSuccess) return err;
  list.run = 1;
  return list_launches<N>(list, adamw_kernel<N, kAnyCodes, FULL>, n, t, sm_count, s, [](const sffn_adamw_tensor& a) { return what_of(a) == kAnyCodes; }, fill);
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
  uint32_t pieces, run;
  ValueEntry e[N];
};

template <int N>
__global__ void __launch_bounds__(kStepThreads) adamw_values_kernel(const __grid_constant__ ValueList<N> list) {
  const int lane = threadIdx.x & 31;
  const uint32_t warps = gridDim.x * (kStepThreads / 32);
  pdl_launch_dependents();
  pdl_wait();
  int e = 0;
  for (uint32_t piece = blockIdx.x * (kStepThreads / 32) + (threadIdx.x >> 5); piece < list.pieces; piece += warps) {
    advance(list, piece, e);
    const ValueEntry& t = list.e[e];
    const uint32_t group0 = (piece - t.begin) * list.run;
    const long long first = (long long)group0 * kGroup;
    if (t.wide && list.run == 4 && t.n - first >= 4 * kGroup) {  // four groups, every load under way first
      uint2 a[4], b[4];
      float um[4], uv[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long at = first + q * kGroup + lane * kPer;
        if (t.m_out) a[q] = __ldcs(reinterpret_cast<const uint2*>(t.m + at));
        if (t.v_out) b[q] = __ldcs(reinterpret_cast<const uint2*>(t.v + at));
        um[q] = t.m_out ? t.m_scale[group0 + q] : 0.f;
        uv[q] = t.v_out ? t.v_scale[group0 + q] : 0.f;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const long long at = first + q * kGroup + lane * kPer;
        f2 f[4];
        if (t.m_out) {
          codes_m(a[q].x, both(unit_m(um[q])), f);
          codes_m(a[q].y, both(unit_m(um[q])), f + 2);
          st32(t.m_out + at, f);
        }
        if (t.v_out) {
          codes_v(b[q].x, both(unit_v(uv[q])), f);
          codes_v(b[q].y, both(unit_v(uv[q])), f + 2);
          st32(t.v_out + at, f);
        }
      }
    } else {
      const long long end = min(t.n, first + (long long)list.run * kGroup);
      for (long long i = first + lane; i < end; i += 32) {
        if (t.m_out) t.m_out[i] = code_m(t.m[i], unit_m(t.m_scale[i / kGroup]));
        if (t.v_out) t.v_out[i] = code_v(t.v[i], unit_v(t.v_scale[i / kGroup]));
      }
    }
  }
}

template <int N>
cudaError_t value_launches(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, int sm_count, cudaStream_t s) {
  ValueList<N> list;
  list.run = run_of(t, n, sm_count, 4);
  return list_launches<N>(list, adamw_values_kernel<N>, n, t, sm_count, s, [](const sffn_adamw_tensor&) { return true; }, [&](ValueEntry& e, int i) {
    e.m = static_cast<const int8_t*>(t[i].m);
    e.v = static_cast<const uint8_t*>(t[i].v);
    e.m_scale = t[i].m_scale;
    e.v_scale = t[i].v_scale;
    e.m_out = m_out ? m_out[i] : nullptr;
    e.v_out = v_out ? v_out[i] : nullptr;
    e.n = t[i].n;
    e.wide = aligned_to(e.m, 8) && aligned_to(e.v, 8) && aligned_to(e.m_out, 32) && aligned_to(e.v_out, 32);
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
  if (fast_roots(c)) return n <= kShort ? adamw_launches<kShort, false>(t, n, c, sm_count, s) : adamw_launches<kLongStep, false>(t, n, c, sm_count, s);
  return adamw_launches<kLongStep, true>(t, n, c, sm_count, s);
}

cudaError_t launch_adamw_values(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, int sm_count, cudaStream_t s) {
  return n <= kShort ? value_launches<kShort>(t, n, m_out, v_out, sm_count, s) : value_launches<kLongStep>(t, n, m_out, v_out, sm_count, s);
}

}  // namespace sffn
