// The norms before and after a block, with its gate, its residual scale and the residual sum:
//
//     h = resid + scale gate . N(y; post gain),   n = N(h; pre gain),   N(v; gain) = v r(v) . gain,  r(v) = 1 / sqrt(mean v^2 + eps)
//
// and its gradients.  With t = gain_pre . dn, rho = r(h), w = scale gain_post . gate:
//
//     g  = dh + rho t - h rho^3 / D sum(t h)                       (= dresid)
//     dy = r w . g - y r^3 / D sum(w y g)
//     dgain_pre = sum_t dn . h rho,   dgain_post = scale sum_t gate . g . y r,   dgate = scale g . gain_post . y r   (summed as the gate is
//     broadcast)
//
// A row belongs to a warp or to a CTA, whose threads hold it in registers, eight consecutive entries each (or up to four such pieces):
// every input is read once.  The forward pass needs two sums over a row, one after the other.  The backward pass needs one round of
// sums: sum(w y g) is put together from sum(w y dh), sum(w y t) and sum(w y h), which do not wait for sum(t h).
// Gradients of gains and of a channel gate are sums over the rows: a CTA's threads own columns and add up the rows that the CTA
// meets in registers; one line of sums a CTA, which block_columns_kernel adds up in order.
#include "block_kernels.cuh"

#include "common.cuh"

namespace sffn {
namespace {

struct BlockParams {
  int T, D;
  int y_bf16, h_bf16, n_bf16, gate_kind;
  const char *y, *resid, *gate;           // row strides in bytes
  int64_t ld_y, ld_resid, ld_gate;
  const float *post_gain, *pre_gain;
  float scale, eps, inv_d;
  char *h, *n;
  int64_t ld_h, ld_n;
  float* stats;
  // backward
  const char *dh, *dn;
  char *dy, *dresid, *dgate;
  int64_t ld_dh, ld_dn, ld_dy, ld_dresid, ld_dgate;
  float* partial;                         // [2][lines][D], or NULL
  int lines, want_pre, want_c;
};

// Eight entries as they lie in memory (16 bytes of bf16, 32 of fp32; fp32 rows may end after four), and as fp32.
struct Raw {
  uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const char* row, int bf16, int c, int D) {
  Raw r;
  const char* p = row + ((int64_t)c << (bf16 ? 1 : 2));
  r.a = *reinterpret_cast<const uint4*>(p);
  r.b = make_uint4(0, 0, 0, 0);
  if (!bf16 && c + 4 < D) r.b = *reinterpret_cast<const uint4*>(p + 16);
  return r;
}
__device__ __forceinline__ void unpack(const Raw& r, int bf16, float* f) {
  if (bf16) {
    Elem<__nv_bfloat16>::unpack(r.a, f);
  } else {
    Elem<float>::unpack(r.a, f);
    Elem<float>::unpack(r.b, f + 4);
  }
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store8(char* row, int bf16, int c, int D, const float* f) {
  char* p = row + ((int64_t)c << (bf16 ? 1 : 2));
  if (bf16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    if (c + 4 < D) *reinterpret_cast<float4*>(p + 16) = make_float4(f[4], f[5], f[6], f[7]);
  }
}
// Eight numbers of a row of D floats that all rows share.
__device__ __forceinline__ void load_gain(const float* g, int c, int D, float* f) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(g + c));
  const float4 b = c + 4 < D ? __ldg(reinterpret_cast<const float4*>(g + c + 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}

// Sums over the W warps of a row, every thread's result bitwise the same.  `room`: W floats, not in use by the sum before.
template <int W>
__device__ __forceinline__ float row_sum(float v, float* room) {
  v = warp_sum(v);
  if constexpr (W == 1) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) room[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < W ? room[lane] : 0.f;
  return warp_sum(v);
}

// W: warps of a row.  V: pieces of eight entries of a thread.  kRows: rows of a CTA.
template <int W, int V>
struct Shape {
  static constexpr int kRows = W == 1 ? 4 : 1, kThreads = 32 * W * kRows;
};

template <int W, int V>
__global__ void __launch_bounds__(Shape<W, V>::kThreads) block_forward_kernel(const __grid_constant__ BlockParams p) {
  __shared__ float room[2][32];
  const int in_row = threadIdx.x % (32 * W), t = blockIdx.x * Shape<W, V>::kRows + threadIdx.x / (32 * W);
  pdl_launch_dependents();
  pdl_wait();
  if (W == 1 && t >= p.T) return;  // (a warp by itself; else a CTA is a row)
  const bool post = p.post_gain != nullptr, pre = p.pre_gain != nullptr;
  Raw y[V], x[V], gate[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = 8 * (in_row + 32 * W * i);
    if (c >= p.D) continue;
    if (p.y) y[i] = load_raw(p.y + t * p.ld_y, p.y_bf16, c, p.D);
    if (p.resid) x[i] = load_raw(p.resid + t * p.ld_resid, p.h_bf16, c, p.D);
    if (p.gate_kind == SFFN_BLOCK_GATE_FULL) gate[i] = load_raw(p.gate + t * p.ld_gate, p.h_bf16, c, p.D);
  }
  float r = 1.f;
  if (post) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (8 * (in_row + 32 * W * i) >= p.D) continue;
      float f[8];
      unpack(y[i], p.y_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(f[j], f[j], ss);
    }
    r = rsqrtf(fmaf(row_sum<W>(ss, room[0]), p.inv_d, p.eps));
  }
  const float factor = p.scale * r * (p.gate_kind == SFFN_BLOCK_GATE_TOKEN ? reinterpret_cast<const float*>(p.gate)[t] : 1.f);
  float h[V][8], hh = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = 8 * (in_row + 32 * W * i);
    if (c >= p.D) continue;
    if (p.resid) unpack(x[i], p.h_bf16, h[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = 0.f;
    if (p.y) {
      float f[8], g[8];
      unpack(y[i], p.y_bf16, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] *= factor;
      if (post) {
        load_gain(p.post_gain, c, p.D, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= g[j];
      }
      if (p.gate_kind == SFFN_BLOCK_GATE_CHANNEL) {
        load_gain(reinterpret_cast<const float*>(p.gate), c, p.D, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= g[j];
      } else if (p.gate_kind == SFFN_BLOCK_GATE_FULL) {
        unpack(gate[i], p.h_bf16, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= g[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] += f[j];
      store8(p.h + t * p.ld_h, p.h_bf16, c, p.D, h[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) hh = fmaf(h[i][j], h[i][j], hh);
  }
  float rho = 0.f;
  if (pre) {
    rho = rsqrtf(fmaf(row_sum<W>(hh, room[1]), p.inv_d, p.eps));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = 8 * (in_row + 32 * W * i);
      if (c >= p.D) continue;
      float g[8];
      load_gain(p.pre_gain, c, p.D, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= h[i][j] * rho;
      store8(p.n + t * p.ld_n, p.n_bf16, c, p.D, g);
    }
  }
  if (p.stats && in_row == 0) {
    p.stats[t] = post ? r : 0.f;
    p.stats[p.T + t] = rho;
  }
}

// Four sums over the W warps of a row.  `room`: 4 W floats, not in use by the sums before.
template <int W>
__device__ __forceinline__ void row_sums(float (&v)[4], float* room) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = warp_sum(v[k]);
  if constexpr (W > 1) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) *reinterpret_cast<float4*>(room + 4 * (threadIdx.x >> 5)) = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    float s = 0.f;  // lane l: sum l % 4, of every eighth warp
#pragma unroll
    for (int w = 0; w < W; w += 8)
      if (w + (lane >> 2) < W) s += room[4 * w + lane];
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = __shfl_sync(0xffffffffu, s, k);
  }
}

// Rows of up to 8192 entries: W warps, two pieces of eight entries a thread (one where W is 1: eight rows a CTA).  Wider ones: 32 warps of up
// to four, whose sums of columns do not fit registers beside the rest.
template <int W, int V>
struct BackShape {
  static constexpr int kRows = W == 1 ? 8 : 1, kThreads = 32 * W * kRows;
  static constexpr int kPerSm = kThreads >= 512 ? 1 : 512 / kThreads;
  static constexpr bool kRing = W < 32;  // rows come through shared memory, which has no room for wider ones
};
constexpr int kBackStages = 4;  // rows under way, at most

__device__ __forceinline__ void copy16(uint32_t to, const char* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t from) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
  return v;
}

// Every thread copies what it will read itself into shared memory, `stages` rows ahead: its own copies are all that it waits for.
// ALL_BF16: y, h and n are bf16, else each is what the call says.
template <int W, int V, bool ALL_BF16>
__global__ void __launch_bounds__(BackShape<W, V>::kThreads, BackShape<W, V>::kPerSm)
    block_backward_kernel(const __grid_constant__ BlockParams p, int stages) {
  constexpr int kRows = BackShape<W, V>::kRows, kThreads = BackShape<W, V>::kThreads;
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ __align__(16) float room[2][4 * W];
  __shared__ float lines[W == 1 ? kRows : 1][W == 1 ? 256 * V : 1];
  const int in_row = threadIdx.x % (32 * W);
  const bool y_bf16 = ALL_BF16 || p.y_bf16, h_bf16 = ALL_BF16 || p.h_bf16, n_bf16 = ALL_BF16 || p.n_bf16;
  const bool post = p.post_gain != nullptr, full = p.gate_kind == SFFN_BLOCK_GATE_FULL, channel = p.gate_kind == SFFN_BLOCK_GATE_CHANNEL;
  const bool has_dh = p.dh != nullptr, has_n = p.dn != nullptr, has_y = p.y != nullptr;
  // The ring: for every stage, array and piece (and half of an fp32 piece) a plane of 16 bytes a thread.
  const int wide_h = h_bf16 ? 1 : 2, wide_n = n_bf16 ? 1 : 2, wide_y = y_bf16 ? 1 : 2;
  struct Array {
    const char* p;
    int64_t ld;
    int plane;
    bool bf16;
  };
  const Array dh = {p.dh, p.ld_dh, 0, h_bf16}, dn = {p.dn, p.ld_dn, has_dh ? wide_h : 0, n_bf16}, h = {p.h, p.ld_h, dn.plane + (has_n ? wide_n : 0), h_bf16};
  const Array y = {p.y, p.ld_y, h.plane + (has_n ? wide_h : 0), y_bf16}, gate = {p.gate, p.ld_gate, y.plane + (has_y ? wide_y : 0), h_bf16};
  const int stage_bytes = (gate.plane + (full ? wide_h : 0)) * V * kThreads * 16;
  const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(ring_raw)) + threadIdx.x * 16;
  auto plane = [&](int stage, const Array& a, int i) { return ring + stage * stage_bytes + (a.plane * V + (a.bf16 ? i : 2 * i)) * (kThreads * 16); };

  pdl_launch_dependents();
  pdl_wait();
  auto copy_piece = [&](int stage, const Array& a, int t, int i, int c) {
    const uint32_t to = plane(stage, a, i);
    const char* from = a.p + t * a.ld + ((int64_t)c << (a.bf16 ? 1 : 2));
    copy16(to, from);
    if (!a.bf16 && c + 4 < p.D) copy16(to + kThreads * 16, from + 16);
  };
  auto fetch = [&](int stage, int t) {
    if constexpr (!BackShape<W, V>::kRing) return;
    if (t < p.T) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = 8 * (in_row + 32 * W * i);
        if (c >= p.D) continue;
        if (has_dh) copy_piece(stage, dh, t, i, c);
        if (has_n) {
          copy_piece(stage, dn, t, i, c);
          copy_piece(stage, h, t, i, c);
        }
        if (has_y) copy_piece(stage, y, t, i, c);
        if (full) copy_piece(stage, gate, t, i, c);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");  // a group a row, empty or not
  };
  auto get = [&](int stage, const Array& a, int t, int i, int c, float* f) {
    Raw r;
    if constexpr (BackShape<W, V>::kRing) {
      const uint32_t from = plane(stage, a, i);
      r.a = shared16(from);
      if (!a.bf16) r.b = c + 4 < p.D ? shared16(from + kThreads * 16) : make_uint4(0, 0, 0, 0);
    } else {
      r = load_raw(a.p + t * a.ld, a.bf16, c, p.D);
    }
    unpack(r, a.bf16, f);
  };

  const int first = blockIdx.x * kRows + threadIdx.x / (32 * W), step = gridDim.x * kRows;
  for (int q = 0; q < stages; ++q) fetch(q, first + q * step);  // (not more than 2^30 rows and a grid's: no overflow)
  // This thread's columns: n's gains, and what multiplies y's entries but for r and a gate of a token's or an entry's.
  float pre[V][8], w[V][8], acc_pre[V][8], acc_c[V][8];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = 8 * (in_row + 32 * W * i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc_pre[i][j] = acc_c[i][j] = pre[i][j] = 0.f;
      w[i][j] = p.scale;
    }
    if (c >= p.D) continue;
    if (has_n) load_gain(p.pre_gain, c, p.D, pre[i]);
    float f[8];
    if (post) {
      load_gain(p.post_gain, c, p.D, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] *= f[j];
    }
    if (channel) {
      load_gain(reinterpret_cast<const float*>(p.gate), c, p.D, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] *= f[j];
    }
  }
  int turn = 0, stage = 0;
  for (int t = first; t < p.T; t += step, turn ^= 1) {
    if (stages >= 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
    const float r = post ? p.stats[t] : 1.f, rho = has_n ? p.stats[p.T + t] : 0.f;
    const float token = p.gate_kind == SFFN_BLOCK_GATE_TOKEN ? reinterpret_cast<const float*>(p.gate)[t] : 1.f;
    float sums[4] = {0.f, 0.f, 0.f, 0.f};  // of t h, w y dh, w y t, w y h
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = 8 * (in_row + 32 * W * i);
      if (c >= p.D) continue;
      float a[8], b[8], e[8];
      if (has_n) {
        get(stage, dn, t, i, c, a);
        get(stage, h, t, i, c, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          a[j] *= pre[i][j];
          sums[0] = fmaf(a[j], b[j], sums[0]);
        }
      }
      if (has_y) {
        get(stage, y, t, i, c, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] *= w[i][j];
        if (full) {
          float f[8];
          get(stage, gate, t, i, c, f);
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] *= f[j];
        }
        if (has_n) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sums[2] = fmaf(e[j], a[j], sums[2]);
            sums[3] = fmaf(e[j], b[j], sums[3]);
          }
        }
        if (has_dh) {
          get(stage, dh, t, i, c, a);
#pragma unroll
          for (int j = 0; j < 8; ++j) sums[1] = fmaf(e[j], a[j], sums[1]);
        }
      }
    }
    row_sums<W>(sums, room[turn]);
    const float k1 = rho * rho * rho * p.inv_d * sums[0];
    const float wyg = fmaf(rho, sums[2], sums[1]) - k1 * sums[3];
    const float k2 = post ? r * r * r * p.inv_d * token * wyg : 0.f, up = r * token, own = p.scale * r * token;
    if (p.dgate && p.gate_kind == SFFN_BLOCK_GATE_TOKEN && in_row == 0) reinterpret_cast<float*>(p.dgate)[t] = r * wyg;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = 8 * (in_row + 32 * W * i);
      if (c >= p.D) continue;
      float g[8], f[8], e[8];
      if (has_dh) get(stage, dh, t, i, c, g);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 0.f;
      if (has_n) {
        get(stage, dn, t, i, c, f);
        get(stage, h, t, i, c, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[j] *= rho;
          g[j] = fmaf(-k1, e[j], fmaf(f[j], pre[i][j], g[j]));
          acc_pre[i][j] = fmaf(f[j], e[j], acc_pre[i][j]);
        }
      }
      if (p.dresid) store8(p.dresid + t * p.ld_dresid, h_bf16, c, p.D, g);
      if (has_y) {
        get(stage, y, t, i, c, f);
        if (full) {
          get(stage, gate, t, i, c, e);
          if (p.dgate) {
            float d[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = up * w[i][j] * g[j] * f[j];
            store8(p.dgate + t * p.ld_dgate, h_bf16, c, p.D, d);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] *= e[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc_c[i][j] = fmaf(own * g[j], f[j], acc_c[i][j]);
        if (p.dy) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = fmaf(up * w[i][j], g[j], -k2 * f[j]);
          store8(p.dy + t * p.ld_dy, y_bf16, c, p.D, f);
        }
      }
    }
    fetch(stage, t + stages * step);  // what was in this stage has been used
    if (++stage == stages) stage = 0;
  }
  // This CTA's line of column sums.
  float* const line = p.partial + (int64_t)blockIdx.x * p.D;
  auto leave = [&](float* to, float (&acc)[V][8]) {
    if constexpr (W > 1) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int c = 8 * (in_row + 32 * W * i);
        if (c < p.D) store8(reinterpret_cast<char*>(to), 0, c, p.D, acc[i]);
      }
    } else {  // of its warps' sums, in their order
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) lines[threadIdx.x >> 5][256 * i + 8 * in_row + j] = acc[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < p.D; c += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < kRows; ++q) s += lines[q][c];
        to[c] = s;
      }
    }
  };
  if (p.want_pre) leave(line, acc_pre);
  if (p.want_c) leave(line + (int64_t)p.lines * p.D, acc_c);
}

// Column sums of `n` lines, added up in order: runs of lines, then the runs.  What the second array holds is sum g y (r, scale, and a
// gate that is not one of the channels in it): times the channel gate it is the post gain's gradient, times the post gain the gate's.
constexpr int kColumnRuns = 32;
__global__ void __launch_bounds__(32 * kColumnRuns) block_columns_kernel(const float* partial, int n, int room, int D, const float* post_gain, const float* gate, float* dpre,
                                                                        float* dpost, float* dgate) {
  __shared__ float sums[kColumnRuns][32];
  pdl_launch_dependents();
  pdl_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5, which = blockIdx.y;
  if (which == 0 ? !dpre : !dpost && !dgate) return;
  float s = 0.f;
  if (c < D) {
    const float* from = partial + (int64_t)which * room * D + c;
    const int first = n * run / kColumnRuns, end = n * (run + 1) / kColumnRuns;
#pragma unroll 8
    for (int l = first; l < end; ++l) s += __ldcg(from + (int64_t)l * D);
  }
  sums[run][threadIdx.x & 31] = s;
  __syncthreads();
  if (run != 0 || c >= D) return;
  s = 0.f;
#pragma unroll
  for (int q = 0; q < kColumnRuns; ++q) s += sums[q][threadIdx.x];
  if (which == 0) {
    dpre[c] = s;
  } else {
    const float gain = post_gain ? post_gain[c] : 1.f, open = gate ? gate[c] : 1.f;
    if (dpost) dpost[c] = s * open;
    if (dgate) dgate[c] = s * gain;
  }
}

BlockParams params_of(const sffn_block_norm& b) {
  BlockParams p{};
  auto bytes = [](int dtype, int64_t ld) { return ld * (dtype == SFFN_BF16 ? 2 : 4); };
  p.T = b.T; p.D = b.D;
  p.y_bf16 = b.y_dtype == SFFN_BF16; p.h_bf16 = b.h_dtype == SFFN_BF16; p.n_bf16 = b.n_dtype == SFFN_BF16;
  p.gate_kind = b.y ? b.gate_kind : SFFN_BLOCK_GATE_NONE;
  p.y = static_cast<const char*>(b.y); p.ld_y = bytes(b.y_dtype, b.ld_y);
  p.resid = static_cast<const char*>(b.resid); p.ld_resid = bytes(b.h_dtype, b.ld_resid);
  p.gate = static_cast<const char*>(b.gate); p.ld_gate = bytes(b.h_dtype, b.ld_gate);
  p.post_gain = b.y ? b.post_gain : nullptr; p.pre_gain = b.pre_gain;
  p.scale = b.scale; p.eps = b.eps; p.inv_d = 1.f / (float)b.D;
  p.h = static_cast<char*>(b.h); p.ld_h = bytes(b.h_dtype, b.ld_h);
  p.n = static_cast<char*>(b.n); p.ld_n = bytes(b.n_dtype, b.ld_n);
  p.stats = b.stats;
  return p;
}

template <int W, int V>
cudaError_t forward(const BlockParams& p, cudaStream_t s) {
  using S = Shape<W, V>;
  return launch_pdl(block_forward_kernel<W, V>, dim3((p.T + S::kRows - 1) / S::kRows), dim3(S::kThreads), 0, s, p);
}
constexpr int kSmShared = 200 * 1024;  // of an SM, for the rings of the CTAs on it (up to eight, with up to 9 KB more each)

template <int W, int V, bool ALL_BF16>
cudaError_t backward(const BlockParams& p, int sm_count, int* lines, cudaStream_t s) {
  using S = BackShape<W, V>;
  static unsigned long long configured = 0;
  cudaError_t e = allow_dynamic_smem(block_backward_kernel<W, V, ALL_BF16>, kSmShared, configured);
  if (e != cudaSuccess) return e;
  const int h = p.h_bf16 ? 1 : 2, n = p.n_bf16 ? 1 : 2, y = p.y_bf16 ? 1 : 2;
  const int planes = (p.dh ? h : 0) + (p.dn ? n + h : 0) + (p.y ? y : 0) + (p.gate_kind == SFFN_BLOCK_GATE_FULL ? h : 0);
  const int stage = S::kRing ? planes * V * S::kThreads * 16 : 0, rows = (p.T + S::kRows - 1) / S::kRows;
  // At most five arrays of fp32, two pieces of 512 threads of an SM: 160 KB.
  int stages = stage > 0 ? kSmShared / S::kPerSm / stage : 1;
  stages = stages > kBackStages ? kBackStages : stages;
  const int room = S::kPerSm * sm_count;
  *lines = rows < room ? rows : room;
  if (*lines > p.lines) *lines = p.lines;
  return launch_pdl(block_backward_kernel<W, V, ALL_BF16>, dim3(*lines), dim3(S::kThreads), (size_t)stages * stage, s, p, stages);
}
template <int W, int V>
cudaError_t backward(const BlockParams& p, int sm_count, int* lines, cudaStream_t s) {
  return p.y_bf16 && p.h_bf16 && p.n_bf16 ? backward<W, V, true>(p, sm_count, lines, s) : backward<W, V, false>(p, sm_count, lines, s);
}

}  // namespace

cudaError_t launch_block_forward(const sffn_block_norm& b, cudaStream_t s) {
  const BlockParams p = params_of(b);
  const bool few = p.T <= 148;  // rows that do not fill the device: as many threads a row as it has pieces
  if (p.D <= 256) return forward<1, 1>(p, s);
  if (p.D <= 1024 && few) return forward<4, 1>(p, s);
  if (p.D <= 512) return forward<1, 2>(p, s);
  if (p.D <= 1024) return forward<1, 4>(p, s);
  if (p.D <= 2048) return few ? forward<8, 1>(p, s) : forward<4, 2>(p, s);
  if (p.D <= 4096) return few ? forward<16, 1>(p, s) : forward<8, 2>(p, s);
  if (p.D <= 8192) return few ? forward<32, 1>(p, s) : forward<16, 2>(p, s);
  if (p.D <= 16384) return forward<32, 2>(p, s);
  return forward<32, 4>(p, s);
}

cudaError_t launch_block_backward(const sffn_block_norm& b, const sffn_block_grads& g, float* partial, int sm_count, cudaStream_t s) {
  BlockParams p = params_of(b);
  auto bytes = [](int dtype, int64_t ld) { return ld * (dtype == SFFN_BF16 ? 2 : 4); };
  p.dh = static_cast<const char*>(g.dh); p.ld_dh = bytes(b.h_dtype, g.ld_dh);
  p.dn = static_cast<const char*>(g.dn); p.ld_dn = bytes(b.n_dtype, g.ld_dn);
  p.dy = static_cast<char*>(g.dy); p.ld_dy = bytes(b.y_dtype, g.ld_dy);
  p.dresid = static_cast<char*>(g.dresid); p.ld_dresid = bytes(b.h_dtype, g.ld_dresid);
  p.dgate = p.gate_kind == SFFN_BLOCK_GATE_TOKEN || p.gate_kind == SFFN_BLOCK_GATE_FULL ? static_cast<char*>(g.dgate) : nullptr;
  p.ld_dgate = bytes(b.h_dtype, g.ld_dgate);
  p.partial = partial;
  p.lines = block_lines(p.D);
  float* const dchannel = p.gate_kind == SFFN_BLOCK_GATE_CHANNEL ? static_cast<float*>(g.dgate) : nullptr;
  p.want_pre = g.dpre_gain != nullptr;
  p.want_c = g.dpost_gain != nullptr || dchannel != nullptr;
  int lines = 0;
  cudaError_t e;
  if (p.D <= 256) e = backward<1, 1>(p, sm_count, &lines, s);
  else if (p.D <= 512) e = backward<2, 1>(p, sm_count, &lines, s);
  else if (p.D <= 1024) e = backward<2, 2>(p, sm_count, &lines, s);
  else if (p.D <= 2048) e = backward<4, 2>(p, sm_count, &lines, s);
  else if (p.D <= 4096) e = backward<8, 2>(p, sm_count, &lines, s);
  else if (p.D <= 8192) e = backward<16, 2>(p, sm_count, &lines, s);
  else if (p.D <= 16384) e = backward<32, 2>(p, sm_count, &lines, s);
  else e = backward<32, 4>(p, sm_count, &lines, s);
  if (e != cudaSuccess || (!p.want_pre && !p.want_c)) return e;
  return launch_pdl(block_columns_kernel, dim3((p.D + 31) / 32, 2), dim3(32 * kColumnRuns), 0, s, (const float*)partial, lines, p.lines, p.D, p.post_gain,
                    p.gate_kind == SFFN_BLOCK_GATE_CHANNEL ? reinterpret_cast<const float*>(p.gate) : (const float*)nullptr, g.dpre_gain, g.dpost_gain, dchannel);
}

}  // namespace sffn
