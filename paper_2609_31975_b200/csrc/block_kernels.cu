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
// A row belongs to a warp or to a CTA, whose threads hold it in registers, eight consecutive entries each (or up to four such pieces), or,
// where there are many of them, in a ring in shared memory: every input is read from memory once up to 8192 columns.  Wider rows have no ring, and
// the backward pass reads them twice, the second time out of L2 where they are still there.  The forward pass needs two sums over a row, one after the other.  The backward pass needs one round of
// sums: sum(w y g) is put together from sum(w y dh), sum(w y t) and sum(w y h), which do not wait for sum(t h).
// Gradients of gains and of a channel gate are sums over the rows: a CTA's threads own columns and add up the rows that the CTA
// meets in registers; one line of sums a CTA, which block_columns_kernel adds up in order.
// Forward, 8192 x 8192, fp32 stream, bf16 y and n, a gate of channels: 131 to 137 us, 5.9 to 6.1 TB/s, bound by memory; 1000 x 4096 in bf16 10 us (33 MB, out of
// L2): 1000 CTAs, four an SM, are 1.7 rounds, each of which reads the gains and the gate again, issue slots 57 %; a row of 4096 3 us, bound by
// the launch and two sums one after the other.  Backward, 4096 x 4096 in bf16: 44 us (201 MB, 4.6 TB/s; issue slots 55 %: each array is
// unpacked twice a row) and 7 for the sums of columns; 5000 x 3840 with an fp32 stream and a gate of tokens: 76 us with them (346 MB, 4.6 TB/s).
// Without a ring, 4096 x 16384 in bf16: forward 155 us (3.5 TB/s), backward 337 (2.4 TB/s; 64 registers a thread, the rest spilled).
#include "block_kernels.cuh"

#include "common.cuh"

namespace sffn {
namespace {

// What becomes of the sums of columns.  The second array holds sum g y (r, scale, and a gate that is not one of the channels in it): times the
// channel gate it is the post gain's gradient, times the post gain the gate's.
struct ColumnSums {
  const float *post_gain, *gate;  // gate: of channels, or NULL
  float *dpre, *dpost, *dgate;    // NULL: not wanted
};
__device__ __forceinline__ void column_out(const ColumnSums& o, int which, int c, float s) {
  if (which == 0) {
    o.dpre[c] = s;
  } else {
    if (o.dpost) o.dpost[c] = s * (o.gate ? o.gate[c] : 1.f);
    if (o.dgate) o.dgate[c] = s * (o.post_gain ? o.post_gain[c] : 1.f);
  }
}

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
  int wide;                               // fp32 rows start on 32 bytes, all of them
  int wide_lines;                         // lines of column sums, likewise
  int together;                           // the launch is one cluster
  ColumnSums sums;
};

// Eight entries as they lie in memory (16 bytes of bf16, 32 of fp32; fp32 rows may end after four), and as fp32.
struct Raw {
  uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const char* row, int bf16, int wide, int c, int D) {
  Raw r;
  const char* p = row + ((int64_t)c << (bf16 ? 1 : 2));
  if (!bf16 && wide && c + 4 < D) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.a.x), "=r"(r.a.y), "=r"(r.a.z), "=r"(r.a.w), "=r"(r.b.x), "=r"(r.b.y), "=r"(r.b.z), "=r"(r.b.w)
                 : "l"(p)
                 : "memory");
    return r;
  }
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
__device__ __forceinline__ void store8(char* row, int bf16, int wide, int c, int D, const float* f) {
  char* p = row + ((int64_t)c << (bf16 ? 1 : 2));
  if (bf16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
  } else if (wide && c + 4 < D) {  // (16 bytes at a time would write every sector of L2 twice)
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7])
                 : "memory");
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

// The same eight entries in pairs, for arithmetic on two at a time.
struct Eight {
  float2 v[4];
};
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 both(float s) { return make_float2(s, s); }
__device__ __forceinline__ Eight operator*(const Eight& a, const Eight& b) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = mul2(a.v[i], b.v[i]);
  return r;
}
__device__ __forceinline__ Eight operator*(const Eight& a, float s) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = mul2(a.v[i], both(s));
  return r;
}
__device__ __forceinline__ Eight fma8(const Eight& a, const Eight& b, const Eight& c) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = fma2(a.v[i], b.v[i], c.v[i]);
  return r;
}
__device__ __forceinline__ Eight fma8(const Eight& a, float s, const Eight& c) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = fma2(a.v[i], both(s), c.v[i]);
  return r;
}
__device__ __forceinline__ Eight eight_of(float s) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = both(s);
  return r;
}
// sum + a . b, the two halves of the sum apart
__device__ __forceinline__ float2 dot8(const Eight& a, const Eight& b, float2 sum) {
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = fma2(a.v[i], b.v[i], sum);
  return sum;
}
__device__ __forceinline__ Eight unpack8(const Raw& r, int bf16) {
  float f[8];
  unpack(r, bf16, f);
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.v[i] = make_float2(f[2 * i], f[2 * i + 1]);
  return e;
}
__device__ __forceinline__ Eight gain8(const float* g, int c, int D) {
  float f[8];
  load_gain(g, c, D, f);
  Eight e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e.v[i] = make_float2(f[2 * i], f[2 * i + 1]);
  return e;
}
__device__ __forceinline__ void store8(char* row, int bf16, int wide, int c, int D, const Eight& e) {
  const float f[8] = {e.v[0].x, e.v[0].y, e.v[1].x, e.v[1].y, e.v[2].x, e.v[2].y, e.v[3].x, e.v[3].y};
  store8(row, bf16, wide, c, D, f);
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
    if (p.y) y[i] = load_raw(p.y + t * p.ld_y, p.y_bf16, p.wide, c, p.D);
    if (p.resid) x[i] = load_raw(p.resid + t * p.ld_resid, p.h_bf16, p.wide, c, p.D);
    if (p.gate_kind == SFFN_BLOCK_GATE_FULL) gate[i] = load_raw(p.gate + t * p.ld_gate, p.h_bf16, p.wide, c, p.D);
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
      store8(p.h + t * p.ld_h, p.h_bf16, p.wide, c, p.D, h[i]);
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
      store8(p.n + t * p.ld_n, p.n_bf16, p.wide, c, p.D, g);
    }
  }
  if (p.stats && in_row == 0) {
    p.stats[t] = post ? r : 0.f;
    p.stats[p.T + t] = rho;
  }
}

// ---- rows through shared memory ---------------------------------------------------------------------------------------

// Four sums over the W warps of a row: six exchanges leave sum k in lanes 8 k to 8 k + 7.  `room`: 4 W floats, not in use by the sums before.
template <int W>
__device__ __forceinline__ void row_sums(float (&v)[4], float* room) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int width = 2; width >= 1; width >>= 1) {
    const bool upper = lane & (8 * width);
#pragma unroll
    for (int i = 0; i < width; ++i) {
      const float send = upper ? v[i] : v[i + width], keep = upper ? v[i + width] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, 8 * width);
    }
  }
  float s = v[0];
#pragma unroll
  for (int o = 4; o >= 1; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if constexpr (W > 1) {
    const int warp = (threadIdx.x >> 5) % W;
    if ((lane & 7) == 0) room[4 * warp + (lane >> 3)] = s;
    __syncthreads();
    s = 0.f;  // lane l: sum l / 8, of every eighth warp
#pragma unroll
    for (int w = 0; w < W; w += 8)
      if (w + (lane & 7) < W) s += room[4 * (w + (lane & 7)) + (lane >> 3)];
#pragma unroll
    for (int o = 1; o <= 4; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = __shfl_sync(0xffffffffu, s, 8 * k);
}

constexpr int kMostStages = 6;         // rows under way, at most
constexpr int kSmShared = 200 * 1024;  // of an SM's shared memory, for the rings of the CTAs on it

// Rows of up to 8192 entries: W warps, one or two pieces of eight entries a thread (W 1: eight rows a CTA).  Wider ones: 32 warps of up to four
// pieces, which have no room in shared memory and whose sums of columns do not fit registers beside the rest.
template <int W, int V>
struct Ring {
  static constexpr int kRows = W == 1 ? 8 : 1, kThreads = 32 * W * kRows;
  static constexpr int kPerSm = kThreads >= 512 ? 1 : 512 / kThreads;
  static constexpr bool kShared = W < 32;
  // Of the backward kernel, beside the ring: sums of a row, of its warps' columns (W 1), statistics of rows (11 KB where W is 1, 6.5 at most elsewhere
  // with a ring).
  static constexpr int kRoom = 2 * 4 * W, kLine = W == 1 ? 256 * V : 1, kStats = 32 * W;
  static constexpr int kStatic = 4 * (kRoom + (W == 1 ? kRows * kLine : 2) + kRows * 3 * kStats);
  static_assert(!kShared || kPerSm * (kSmShared / kPerSm + kStatic + 1024) <= 228 * 1024, "the CTAs of an SM, with the 1 KB that each takes of it by itself");
};
__device__ __forceinline__ void copy16(uint32_t to, const char* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint4 shared16(uint32_t from) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
  return v;
}
// Rows of a matrix; in a ring's stage, its first plane (16 bytes a thread and piece; two of an fp32 matrix).
struct Array {
  const char* p;
  int64_t ld;
  int plane;
  bool bf16;
};
// Every warp copies what it will read itself, `stages` rows ahead, 512 consecutive bytes at a time: its own copies are all that it waits for.
template <int W, int V>
struct Rows {
  static constexpr int kPlane = Ring<W, V>::kThreads * 16;
  uint32_t ring;  // this thread's 16 bytes of the first plane
  int D, T, wide, in_row, stages, stage_bytes;
  __device__ __forceinline__ Rows(const BlockParams& p, const uint8_t* raw, int stages_, int planes)
      : ring(static_cast<uint32_t>(__cvta_generic_to_shared(raw)) + threadIdx.x * 16), D(p.D), T(p.T), wide(p.wide), in_row(threadIdx.x % (32 * W)), stages(stages_),
        stage_bytes(planes * V * kPlane) {}
  __device__ __forceinline__ int column(int i) const { return 8 * (in_row + 32 * W * i); }
  __device__ __forceinline__ uint32_t plane(int stage, const Array& a, int i) const {
    return ring + stage * stage_bytes + (a.plane * V + (a.bf16 ? i : 2 * i)) * kPlane;
  }
  __device__ __forceinline__ void copy(int stage, const Array& a, int t, int i) const {
    if (!a.p) return;
    const int c = column(i);
    const uint32_t to = plane(stage, a, i);
    const char* const row = a.p + t * a.ld;
    if (a.bf16) {
      if (c < D) copy16(to, row + 2 * c);
    } else {  // a warp's 256 columns: four of each lane, and four 128 further on
      const int d = c - 4 * (int)(threadIdx.x & 31);
      if (d < D) copy16(to, row + 4 * d);
      if (d + 128 < D) copy16(to + kPlane, row + 4 * d + 512);
    }
  }
  // A row of each array, one group of copies, empty or not.
  template <typename... A>
  __device__ __forceinline__ void fetch(int stage, int t, const A&... arrays) const {
    if constexpr (Ring<W, V>::kShared) {
      __syncwarp();  // all lanes have read what was there
      if (t < T) {
#pragma unroll
        for (int i = 0; i < V; ++i) (copy(stage, arrays, t, i), ...);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  }
  // The oldest row is there, all but `more` of the rows under way.
  __device__ __forceinline__ void wait(int more) const {
    if constexpr (Ring<W, V>::kShared) {
      if (more >= 5) asm volatile("cp.async.wait_group 5;" ::: "memory");
      else if (more == 4) asm volatile("cp.async.wait_group 4;" ::: "memory");
      else if (more == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (more == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
      else if (more == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncwarp();
    }
  }
  __device__ __forceinline__ Eight get(int stage, const Array& a, int t, int i) const {
    const int c = column(i);
    Raw r;
    if constexpr (Ring<W, V>::kShared) {
      const uint32_t at = plane(stage, a, i);
      if (a.bf16) {
        r.a = shared16(at);
      } else {  // lanes 0 to 15 have the first plane's 512 bytes, 32 each; their two reads in turn, so that eight lanes meet all banks
        const int lane = threadIdx.x & 31;
        const uint32_t own = at - 16 * lane + (lane >> 4) * kPlane + 32 * (lane & 15), swap = (lane & 4) << 2;
        const uint4 u = shared16(own + swap), v = shared16(own + (16 ^ swap));
        r.a = swap ? v : u;
        r.b = c + 4 < D ? (swap ? u : v) : make_uint4(0, 0, 0, 0);
      }
    } else {
      r = load_raw(a.p + t * a.ld, a.bf16, wide, c, D);
    }
    return unpack8(r, a.bf16);
  }
};
// What multiplies y's entries in a thread's columns but for r and a gate of a token's or an entry's.
template <int W, int V>
__device__ __forceinline__ void weights_of(const BlockParams& p, const Rows<W, V>& rows, Eight (&w)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    w[i] = eight_of(p.scale);
    const int c = rows.column(i);
    if (c >= p.D) continue;
    if (p.post_gain) w[i] = w[i] * gain8(p.post_gain, c, p.D);
    if (p.gate_kind == SFFN_BLOCK_GATE_CHANNEL) w[i] = w[i] * gain8(reinterpret_cast<const float*>(p.gate), c, p.D);
  }
}

// The forward pass over many rows.  ALL_BF16: y, h and n are bf16, else each is what the call says.
template <int W, int V, bool ALL_BF16>
__global__ void __launch_bounds__(Ring<W, V>::kThreads, Ring<W, V>::kPerSm) block_forward_rows_kernel(const __grid_constant__ BlockParams p, int stages, int planes) {
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ float room[2][32];
  const bool y_bf16 = ALL_BF16 || p.y_bf16, h_bf16 = ALL_BF16 || p.h_bf16, n_bf16 = ALL_BF16 || p.n_bf16;
  const bool post = p.post_gain != nullptr, pre = p.pre_gain != nullptr, full = p.gate_kind == SFFN_BLOCK_GATE_FULL;
  const Rows<W, V> rows(p, ring_raw, stages, planes);
  const Array y = {p.y, p.ld_y, 0, y_bf16}, x = {p.resid, p.ld_resid, p.y ? (y_bf16 ? 1 : 2) : 0, h_bf16};
  const Array gate = {full ? p.gate : nullptr, p.ld_gate, x.plane + (p.resid ? (h_bf16 ? 1 : 2) : 0), h_bf16};
  pdl_launch_dependents();
  pdl_wait();
  const int step = gridDim.x;
  for (int q = 0; q < stages; ++q) rows.fetch(q, blockIdx.x + q * step, y, x, gate);
  Eight w[V], gain[V];
  weights_of(p, rows, w);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    gain[i] = eight_of(0.f);
    if (pre && rows.column(i) < p.D) gain[i] = gain8(p.pre_gain, rows.column(i), p.D);
  }
  int stage = 0, turn = 0;
  for (int t = blockIdx.x; t < p.T; t += step, turn ^= 1) {
    rows.wait(stages - 1);
    float r = 1.f;
    if (post) {
      float2 s = both(0.f);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (rows.column(i) >= p.D) continue;
        const Eight f = rows.get(stage, y, t, i);
        s = dot8(f, f, s);
      }
      r = rsqrtf(fmaf(row_sum<W>(s.x + s.y, room[0]), p.inv_d, p.eps));
    }
    const float factor = r * (p.gate_kind == SFFN_BLOCK_GATE_TOKEN ? reinterpret_cast<const float*>(p.gate)[t] : 1.f);
    Eight h[V];
    float2 s = both(0.f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = rows.column(i);
      if (c >= p.D) continue;
      h[i] = p.resid ? rows.get(stage, x, t, i) : eight_of(0.f);
      if (p.y) {
        Eight f = rows.get(stage, y, t, i) * factor;
        if (full) f = f * rows.get(stage, gate, t, i);
        h[i] = fma8(f, w[i], h[i]);
        store8(p.h + t * p.ld_h, h_bf16, p.wide, c, p.D, h[i]);
      }
      s = dot8(h[i], h[i], s);
    }
    rows.fetch(stage, t + stages * step, y, x, gate);  // what was in this stage has been used
    if (++stage == stages) stage = 0;
    float rho = 0.f;
    if (pre) {  // (a barrier lies between a sum and the one that takes its room)
      rho = rsqrtf(fmaf(row_sum<W>(s.x + s.y, room[post ? 1 : turn]), p.inv_d, p.eps));
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (rows.column(i) < p.D) store8(p.n + t * p.ld_n, n_bf16, p.wide, rows.column(i), p.D, h[i] * rho * gain[i]);
    } else if (post) {
      __syncthreads();
    }
    if (p.stats && threadIdx.x == 0) {
      p.stats[t] = post ? r : 0.f;
      p.stats[p.T + t] = rho;
    }
  }
}

// The backward pass.
template <int W, int V, bool ALL_BF16>
__global__ void __launch_bounds__(Ring<W, V>::kThreads, Ring<W, V>::kPerSm) block_backward_kernel(const __grid_constant__ BlockParams p, int stages, int planes) {
  constexpr int kRows = Ring<W, V>::kRows, kThreads = Ring<W, V>::kThreads;
  extern __shared__ __align__(16) uint8_t ring_raw[];
  using R = Ring<W, V>;
  __shared__ float room[2][R::kRoom / 2];
  __shared__ __align__(8) float lines[W == 1 ? kRows : 1][R::kLine];
  const bool y_bf16 = ALL_BF16 || p.y_bf16, h_bf16 = ALL_BF16 || p.h_bf16, n_bf16 = ALL_BF16 || p.n_bf16;
  const bool post = p.post_gain != nullptr, full = p.gate_kind == SFFN_BLOCK_GATE_FULL;
  const bool has_dh = p.dh != nullptr, has_n = p.dn != nullptr, has_y = p.y != nullptr;
  const int wide_h = h_bf16 ? 1 : 2, wide_n = n_bf16 ? 1 : 2, wide_y = y_bf16 ? 1 : 2;
  const Array dh = {p.dh, p.ld_dh, 0, h_bf16}, dn = {p.dn, p.ld_dn, has_dh ? wide_h : 0, n_bf16}, h = {has_n ? p.h : nullptr, p.ld_h, dn.plane + (has_n ? wide_n : 0), h_bf16};
  const Array y = {p.y, p.ld_y, h.plane + (has_n ? wide_h : 0), y_bf16}, gate = {full ? p.gate : nullptr, p.ld_gate, y.plane + (has_y ? wide_y : 0), h_bf16};
  const Rows<W, V> rows(p, ring_raw, stages, planes);
  pdl_launch_dependents();
  pdl_wait();
  const int first = blockIdx.x * kRows + threadIdx.x / (32 * W), step = gridDim.x * kRows;
  for (int q = 0; q < stages; ++q) rows.fetch(q, first + q * step, dh, dn, h, y, gate);  // (not more than 2^30 rows and a grid's: no overflow)
  Eight pre[V], w[V], acc_pre[V], acc_c[V];
  weights_of(p, rows, w);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    acc_pre[i] = acc_c[i] = pre[i] = eight_of(0.f);
    if (has_n && rows.column(i) < p.D) pre[i] = gain8(p.pre_gain, rows.column(i), p.D);
  }
  // Statistics and a gate of tokens: for as many of its rows as it has threads, a row's warps bring them into shared memory at once.  (A load a
  // row and thread, even one row ahead, costs a fifth: the wait for the ring's copies waits for it too.)
  __shared__ float stat[kRows][3][R::kStats];
  float (*const own_stat)[32 * W] = stat[threadIdx.x / (32 * W)];
  int turn = 0, stage = 0, at_stat = 0;
  for (int t = first; t < p.T; t += step, turn ^= 1) {
    if (at_stat == 0) {  // (what was there has been read: a sum's barrier lies between)
      const int mine = t + rows.in_row * step;
      if (rows.in_row < (p.T - t + step - 1) / step) {
        own_stat[0][rows.in_row] = post ? p.stats[mine] : 1.f;
        own_stat[1][rows.in_row] = has_n ? p.stats[p.T + mine] : 0.f;
        own_stat[2][rows.in_row] = p.gate_kind == SFFN_BLOCK_GATE_TOKEN ? reinterpret_cast<const float*>(p.gate)[mine] : 1.f;
      }
      if constexpr (W == 1) __syncwarp();
      else __syncthreads();
    }
    const float r = own_stat[0][at_stat], rho = own_stat[1][at_stat], token = own_stat[2][at_stat];
    if (++at_stat == 32 * W) at_stat = 0;
    rows.wait(stages - 1);
    // With h' = rho h and y' = r y (of size one, whatever the rows are: cubes of statistics would leave fp32): sums of t h', w y' dh, w y' t, w y' h'
    float2 s[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (rows.column(i) >= p.D) continue;
      Eight a, b;
      if (has_n) {
        a = rows.get(stage, dn, t, i) * pre[i];
        b = rows.get(stage, h, t, i) * rho;
        s[0] = dot8(a, b, s[0]);
      }
      if (has_y) {
        Eight e = rows.get(stage, y, t, i) * r * w[i];
        if (full) e = e * rows.get(stage, gate, t, i);
        if (has_n) {
          s[2] = dot8(e, a, s[2]);
          s[3] = dot8(e, b, s[3]);
        }
        if (has_dh) s[1] = dot8(e, rows.get(stage, dh, t, i), s[1]);
      }
    }
    float sums[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[k] = s[k].x + s[k].y;
    row_sums<W>(sums, room[turn]);
    // g = dh + rho t - k1 h',   sum(w y' g),   dy = up w g - k2 y'
    const float mean = sums[0] * p.inv_d, k1 = rho * mean, wyg = fmaf(rho, fmaf(-mean, sums[3], sums[2]), sums[1]);
    const float up = r * token, k2 = post ? up * wyg * p.inv_d : 0.f, own = p.scale * token;
    if (p.dgate && p.gate_kind == SFFN_BLOCK_GATE_TOKEN && rows.in_row == 0) reinterpret_cast<float*>(p.dgate)[t] = wyg;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = rows.column(i);
      if (c >= p.D) continue;
      Eight g = has_dh ? rows.get(stage, dh, t, i) : eight_of(0.f);
      if (has_n) {
        const Eight f = rows.get(stage, dn, t, i), b = rows.get(stage, h, t, i) * rho;
        g = fma8(b, -k1, fma8(f * rho, pre[i], g));
        acc_pre[i] = fma8(f, b, acc_pre[i]);
      }
      if (p.dresid) store8(p.dresid + t * p.ld_dresid, h_bf16, p.wide, c, p.D, g);
      if (has_y) {
        const Eight f = rows.get(stage, y, t, i) * r;
        if (full) {
          if (p.dgate) store8(p.dgate + t * p.ld_dgate, h_bf16, p.wide, c, p.D, w[i] * g * f);
          g = g * rows.get(stage, gate, t, i);
        }
        acc_c[i] = fma8(g * own, f, acc_c[i]);
        if (p.dy) store8(p.dy + t * p.ld_dy, y_bf16, p.wide, c, p.D, fma8(w[i] * up, g, f * -k2));
      }
    }
    rows.fetch(stage, t + stages * step, dh, dn, h, y, gate);  // what was in this stage has been used
    if (++stage == stages) stage = 0;
  }
  // This CTA's line of column sums.
  float* const line = p.partial + (int64_t)blockIdx.x * p.D;
  auto leave = [&](float* to, const Eight (&acc)[V]) {
    if constexpr (W > 1) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (rows.column(i) < p.D) store8(reinterpret_cast<char*>(to), 0, p.wide_lines, rows.column(i), p.D, acc[i]);
    } else {  // of its warps' sums, in their order
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(&lines[threadIdx.x >> 5][256 * i + 8 * rows.in_row + 2 * j]) = acc[i].v[j];
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
  if (!p.together) return;
  // The whole launch is one cluster: it adds up its lines itself.
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  for (int c = blockIdx.x * kThreads + threadIdx.x; c < 2 * p.D; c += gridDim.x * kThreads) {
    const int which = c >= p.D, column = which ? c - p.D : c;
    if (which ? !p.want_c : !p.want_pre) continue;
    float s = 0.f;
    for (int l = 0; l < gridDim.x; ++l) s += __ldcg(p.partial + ((int64_t)which * p.lines + l) * p.D + column);
    column_out(p.sums, which, column, s);
  }
}

// Column sums of `n` lines, added up in order: runs of lines, then the runs.
constexpr int kColumnRuns = 32;
__global__ void __launch_bounds__(32 * kColumnRuns) block_columns_kernel(const float* partial, int n, int room, int D, const ColumnSums out) {
  __shared__ float sums[kColumnRuns][32];
  pdl_launch_dependents();
  pdl_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5, which = blockIdx.y;
  if (which == 0 ? !out.dpre : !out.dpost && !out.dgate) return;
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
  column_out(out, which, c, s);
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
  p.wide = 1;
  auto look = [&](const void* at, int64_t ld, bool bf16) { p.wide = p.wide && (bf16 || !at || ((reinterpret_cast<uintptr_t>(at) | ld) & 31) == 0); };
  look(p.y, p.ld_y, p.y_bf16);
  look(p.resid, p.ld_resid, p.h_bf16);
  look(p.h, p.ld_h, p.h_bf16);
  look(p.n, p.ld_n, p.n_bf16);
  if (p.gate_kind == SFFN_BLOCK_GATE_FULL) look(p.gate, p.ld_gate, p.h_bf16);
  return p;
}

constexpr int kManyRows = 8;           // rows an SM
// Stages of a ring of so many planes, and its bytes; at most five arrays of fp32, two pieces of 512 threads of an SM: 160 KB a stage.
template <int W, int V>
int stages_of(int planes, size_t* bytes) {
  using S = Ring<W, V>;
  const int stage = S::kShared ? planes * V * S::kThreads * 16 : 0, room = stage > 0 ? kSmShared / S::kPerSm / stage : 1;
  const int stages = room > kMostStages ? kMostStages : room;
  *bytes = (size_t)stages * stage;
  return stages;
}

template <int W, int V>
cudaError_t forward(const BlockParams& p, cudaStream_t s) {
  using S = Shape<W, V>;
  return launch_pdl(block_forward_kernel<W, V>, dim3((p.T + S::kRows - 1) / S::kRows), dim3(S::kThreads), 0, s, p);
}
template <int W, int V, bool ALL_BF16>
cudaError_t forward_rows(const BlockParams& p, int stages, int planes, size_t bytes, int sm_count, cudaStream_t s) {
  static unsigned long long configured = 0;
  const cudaError_t e = allow_dynamic_smem(block_forward_rows_kernel<W, V, ALL_BF16>, kSmShared, configured);
  if (e != cudaSuccess) return e;
  const int room = Ring<W, V>::kPerSm * sm_count;
  return launch_pdl(block_forward_rows_kernel<W, V, ALL_BF16>, dim3(p.T < room ? p.T : room), dim3(Ring<W, V>::kThreads), bytes, s, p, stages, planes);
}
template <int W, int V>
cudaError_t forward_rows(const BlockParams& p, int sm_count, cudaStream_t s) {
  const int h = p.h_bf16 ? 1 : 2, planes = (p.y ? (p.y_bf16 ? 1 : 2) : 0) + (p.resid ? h : 0) + (p.gate_kind == SFFN_BLOCK_GATE_FULL ? h : 0);
  size_t bytes = 0;
  const int stages = stages_of<W, V>(planes, &bytes);
  return p.y_bf16 && p.h_bf16 && p.n_bf16 ? forward_rows<W, V, true>(p, stages, planes, bytes, sm_count, s)
                                          : forward_rows<W, V, false>(p, stages, planes, bytes, sm_count, s);
}
template <int W, int V, bool ALL_BF16>
cudaError_t backward(const BlockParams& p, int sm_count, int* lines, cudaStream_t s) {
  using S = Ring<W, V>;
  static unsigned long long configured = 0;
  cudaError_t e = allow_dynamic_smem(block_backward_kernel<W, V, ALL_BF16>, kSmShared, configured);
  if (e != cudaSuccess) return e;
  const int h = p.h_bf16 ? 1 : 2, n = p.n_bf16 ? 1 : 2, y = p.y_bf16 ? 1 : 2;
  const int planes = (p.dh ? h : 0) + (p.dn ? n + h : 0) + (p.y ? y : 0) + (p.gate_kind == SFFN_BLOCK_GATE_FULL ? h : 0);
  size_t bytes = 0;
  const int stages = stages_of<W, V>(planes, &bytes), rows = (p.T + S::kRows - 1) / S::kRows, room = S::kPerSm * sm_count;
  *lines = rows < room ? rows : room;
  if (*lines > p.lines) *lines = p.lines;
  // So few CTAs that they are a cluster (of eight at most): one launch less (64 tokens of 256: 14.8 / 11.8 us).
  BlockParams q = p;
  q.together = *lines <= 8 && (p.want_pre || p.want_c);
  const cudaError_t launched = launch_clusters(q.together ? *lines : 1, block_backward_kernel<W, V, ALL_BF16>, dim3(*lines), dim3(S::kThreads), bytes, s, q, stages, planes);
  if (q.together) *lines = 0;
  return launched;
}
template <int W, int V>
cudaError_t backward(const BlockParams& p, int sm_count, int* lines, cudaStream_t s) {
  return p.y_bf16 && p.h_bf16 && p.n_bf16 ? backward<W, V, true>(p, sm_count, lines, s) : backward<W, V, false>(p, sm_count, lines, s);
}

}  // namespace

cudaError_t launch_block_forward(const sffn_block_norm& b, int sm_count, cudaStream_t s) {
  const BlockParams p = params_of(b);
  // Rows that do not fill the device: as many threads a row as it has pieces.
  const bool few = p.T <= sm_count;
  // Enough of them for every CTA to have several: through rings.
  const bool many = p.T >= kManyRows * sm_count;
  if (p.D <= 256) return forward<1, 1>(p, s);
  if (p.D <= 1024 && few) return forward<4, 1>(p, s);
  if (p.D <= 512) return forward<1, 2>(p, s);
  if (p.D <= 1024) return forward<1, 4>(p, s);
  if (p.D <= 2048) return few ? forward<8, 1>(p, s) : many ? forward_rows<4, 2>(p, sm_count, s) : forward<4, 2>(p, s);
  if (p.D <= 4096) return few ? forward<16, 1>(p, s) : many ? forward_rows<8, 2>(p, sm_count, s) : forward<8, 2>(p, s);
  if (p.D <= 8192) return few ? forward<32, 1>(p, s) : many ? forward_rows<16, 2>(p, sm_count, s) : forward<16, 2>(p, s);
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
  auto look = [&](const void* at, int64_t ld, bool bf16) { p.wide = p.wide && (bf16 || !at || ((reinterpret_cast<uintptr_t>(at) | ld) & 31) == 0); };
  look(p.dh, p.ld_dh, p.h_bf16);
  look(p.dn, p.ld_dn, p.n_bf16);
  look(p.dy, p.ld_dy, p.y_bf16);
  look(p.dresid, p.ld_dresid, p.h_bf16);
  if (p.gate_kind == SFFN_BLOCK_GATE_FULL) look(p.dgate, p.ld_dgate, p.h_bf16);
  p.partial = partial;
  p.lines = block_lines(p.D);
  p.wide_lines = p.D % 8 == 0 && (reinterpret_cast<uintptr_t>(partial) & 31) == 0;  // (a workspace starts on 16 bytes)
  p.sums = {p.post_gain, p.gate_kind == SFFN_BLOCK_GATE_CHANNEL ? reinterpret_cast<const float*>(p.gate) : nullptr, g.dpre_gain, g.dpost_gain,
            p.gate_kind == SFFN_BLOCK_GATE_CHANNEL ? static_cast<float*>(g.dgate) : nullptr};
  p.want_pre = p.sums.dpre != nullptr;
  p.want_c = p.sums.dpost || p.sums.dgate;
  int lines = 0;
  cudaError_t e;
  if (p.D <= 256) e = backward<1, 1>(p, sm_count, &lines, s);
  else if (p.D <= 512) e = backward<2, 1>(p, sm_count, &lines, s);
  else if (p.D <= 1024) e = backward<4, 1>(p, sm_count, &lines, s);
  else if (p.D <= 2048) e = backward<8, 1>(p, sm_count, &lines, s);
  else if (p.D <= 4096) e = backward<16, 1>(p, sm_count, &lines, s);
  else if (p.D <= 8192) e = backward<16, 2>(p, sm_count, &lines, s);
  else if (p.D <= 16384) e = backward<32, 2>(p, sm_count, &lines, s);
  else e = backward<32, 4>(p, sm_count, &lines, s);
  if (e != cudaSuccess || lines == 0 || (!p.want_pre && !p.want_c)) return e;
  return launch_pdl(block_columns_kernel, dim3((p.D + 31) / 32, 2), dim3(32 * kColumnRuns), 0, s, (const float*)partial, lines, p.lines, p.D, p.sums);
}

}  // namespace sffn
