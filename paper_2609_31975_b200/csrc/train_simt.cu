// Products of small training calls in fp32 FMAs (fp32 storage; larger calls split their operands for the tensor cores).
//
// A CTA owns a 32 x 64 tile of C, or z and u of 32 tokens x 32 neurons; four threads 8 x 4 of it, a quarter of a piece's k each, in packed
// FMAs.  For up to 16 rows: 8 x 64 tiles, eight threads 4 x 4, an eighth of the k each.  Pieces of 64 k go through registers into
// [k][m] and [k][n] arrays, whichever way an operand lies in memory, the next piece under way while one is multiplied.  Such a call has
// few tiles and is bound by latency, so K is cut among up to eight CTAs of a cluster: each leaves its sums in shared memory and takes
// a share of the tile's rows, which it adds up over all of them, in order.
// 64 tokens, 256 x 1024, in a loop: forward 17 us, backward 29, of which launches 4 and 6 (20 and 33 with 4 x 4 a thread, 59 and 114 without
// clusters); 32 tokens, 4096 x 14336, forward 476 us (577), three times the FMAs' time: loads of a piece wait for their stores.  1 token:
// 264 us for 705 MB.
#include "train_kernels.cuh"

namespace sffn {
namespace {

constexpr int kCols = 64, kDepth = 64, kThreads = 256;
constexpr int kMaxSplit = 8;
constexpr int kFewRows = 16;  // up to so many, tiles of 8 rows

// A thread's share of a [kDepth][N] piece: quads of four values, consecutive in memory.
template <int N>
struct Piece {
  static constexpr int kAll = N * kDepth / 4, kQuads = (kAll + kThreads - 1) / kThreads;
  float4 v[kQuads];

  // Quad i of a K-major piece: two lanes take 32 bytes of a row (four 64, of eight rows), a warp sixteen rows, so that its four stores
  // (one a k) meet no bank twice.
  static constexpr int kShare = N < 16 ? 4 : 2, kTall = 32 / kShare;
  __device__ __forceinline__ static int row_of(int i) { return (i >> 5) % (N / kTall) * kTall + (i & 31) / kShare; }
  __device__ __forceinline__ static int k_of(int i) { return ((i >> 5) / (N / kTall) * kShare + i % kShare) * 4; }

  // rows are a multiple of 16 bytes apart; along an axis that ends inside a quad what lies beyond is not looked at
  __device__ __forceinline__ void fetch(const TrainOperand& o, bool major_k, int row0, int rows, int k0, int k1) {
    const float* p = static_cast<const float*>(o.data);
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
      const int i = threadIdx.x + q * kThreads;
      const int r = major_k ? row_of(i) : i % (N / 4) * 4, k = major_k ? k_of(i) : i / (N / 4);
      const int line = major_k ? row0 + r : k0 + k, at = major_k ? k0 + k : row0 + r, lines = major_k ? rows : k1, end = major_k ? k1 : rows;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < kAll && line < lines && at < end) {
        const float* s = p + line * o.ld + at;
        if (at + 4 <= end) {
          f = *reinterpret_cast<const float4*>(s);
        } else {
          f.x = s[0];
          if (at + 1 < end) f.y = s[1];
          if (at + 2 < end) f.z = s[2];
        }
      }
      v[q] = f;
    }
  }
  __device__ __forceinline__ void store(float (*s)[N + 4], bool major_k) const {
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
      const int i = threadIdx.x + q * kThreads;
      if (i >= kAll) continue;
      if (major_k) {
        const int r = row_of(i), k = k_of(i);
        s[k][r] = v[q].x; s[k + 1][r] = v[q].y; s[k + 2][r] = v[q].z; s[k + 3][r] = v[q].w;
      } else {
        *reinterpret_cast<float4*>(&s[i / (N / 4)][i % (N / 4) * 4]) = v[q];
      }
    }
  }
};

__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 remote_quad(const float* local, int rank) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(local)), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(r) : "memory");
  return v;
}

// Four values of a row, the first n of them: rows may end, and start, anywhere in a user's matrix of odd width.
__device__ __forceinline__ void put4(void* base, int64_t at, const float* v, int n) {
  float* p = static_cast<float*>(base) + at;
  if (n == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void get4(const void* base, int64_t at, float* v, int n) {
  const float* p = static_cast<const float*>(base) + at;
  if (n == 4) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}

// A cluster of `splits` CTAs for each tile, tiles along M first (what a short batch has few of: they share the weights' rows in L2),
// then along N, then of the batch.  kRows: 32, or 8 for a handful of tokens, where 32 rows of products would be mostly of zeros.
template <int EPI, int kRows>
__global__ void __launch_bounds__(kThreads) train_simt_kernel(const __grid_constant__ TrainGemm g, int splits) {
  constexpr bool kDual = EPI == kEpiGateUp;
  constexpr int kNeurons = kDual ? kCols / 2 : kCols;  // output columns of a tile
  __shared__ __align__(16) float pool[kDepth * (kRows + 4 + kCols + 4)];
  float(*const sa)[kRows + 4] = reinterpret_cast<float(*)[kRows + 4]>(pool);
  float(*const sb)[kCols + 4] = reinterpret_cast<float(*)[kCols + 4]>(pool + kDepth * (kRows + 4));  // kDual: columns of W_g, then of W_up
  __shared__ __align__(16) float tile[kRows][kCols + 4];
  constexpr int kMine = kRows < 32 ? 4 : 8;  // rows of a thread
  constexpr int kSide = 16 * (kRows / kMine), kParts = kThreads / kSide, kShare = kDepth / kParts;  // threads of a tile; parts of a piece's k
  pdl_launch_dependents();
  pdl_wait();
  const int tx = threadIdx.x & 15, ty = threadIdx.x / 16 % (kRows / kMine), part_k = threadIdx.x / kSide;
  const int m_tiles = (g.M + kRows - 1) / kRows, n_tiles = (g.N + kNeurons - 1) / kNeurons;
  const int at_tile = blockIdx.x / splits, split = blockIdx.x - at_tile * splits, at_col = at_tile / m_tiles, z = at_col / n_tiles;
  const int m0 = (at_tile - at_col * m_tiles) * kRows, n0 = (at_col - z * n_tiles) * kNeurons;
  // K of all parts in a row, in pieces
  const int parts = kDual ? 1 : g.parts, per = (g.K + kDepth - 1) / kDepth, pieces = parts * per;
  const int first = (int)((long long)pieces * split / splits), last = (int)((long long)pieces * (split + 1) / splits);
  float2 acc[kMine][2] = {};
  Piece<kRows> pa;
  Piece<kDual ? kNeurons : kCols> pb;
  Piece<kDual ? kNeurons : kRows> pu;  // kDual: of W_up
  auto fetch = [&](int i) {
    const int part = i / per, k0 = (i - part * per) * kDepth, at = g.batch > 1 ? z : part;
    pa.fetch(g.a[kDual ? 0 : at], g.a_major_k, m0, g.M, k0, g.K);
    pb.fetch(g.b[kDual ? 0 : at], g.b_major_k, n0, g.N, k0, g.K);
    if constexpr (kDual) pu.fetch(g.b[1], g.b_major_k, n0, g.N, k0, g.K);
  };
  auto store = [&]() {
    pa.store(sa, g.a_major_k);
    if constexpr (kDual) {  // always K-major
#pragma unroll
      for (int q = 0; q < Piece<kNeurons>::kQuads; ++q) {
        const int i = threadIdx.x + q * kThreads, r = pb.row_of(i), k = pb.k_of(i);
        sb[k][r] = pb.v[q].x; sb[k + 1][r] = pb.v[q].y; sb[k + 2][r] = pb.v[q].z; sb[k + 3][r] = pb.v[q].w;
        sb[k][kNeurons + r] = pu.v[q].x; sb[k + 1][kNeurons + r] = pu.v[q].y; sb[k + 2][kNeurons + r] = pu.v[q].z; sb[k + 3][kNeurons + r] = pu.v[q].w;
      }
    } else {
      pb.store(sb, g.b_major_k);
    }
  };
  if (first < last) fetch(first);
  for (int i = first; i < last; ++i) {
    store();
    __syncthreads();
    if (i + 1 < last) fetch(i + 1);
    const int left_k = g.K - i % per * kDepth, k_end = min(kShare, left_k - part_k * kShare);  // the last piece of K may be short
#pragma unroll 8
    for (int q = 0; q < k_end; ++q) {
      const int k = part_k * kShare + q;
      const float4 b = *reinterpret_cast<const float4*>(&sb[k][4 * tx]);
      alignas(16) float av[kMine];
#pragma unroll
      for (int i = 0; i < kMine; i += 4) *reinterpret_cast<float4*>(av + i) = *reinterpret_cast<const float4*>(&sa[k][kMine * ty + i]);
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        acc[i][0] = fma2(make_float2(av[i], av[i]), make_float2(b.x, b.y), acc[i][0]);
        acc[i][1] = fma2(make_float2(av[i], av[i]), make_float2(b.z, b.w), acc[i][1]);
      }
    }
    __syncthreads();
  }
  float(*const other)[kRows][kCols + 4] = reinterpret_cast<float(*)[kRows][kCols + 4]>(pool);  // the operands' arrays are free
  static_assert((kParts - 1) * kRows * (kCols + 4) <= kDepth * (kRows + 4 + kCols + 4), "the parts' sums fit the operands' arrays");
  if (part_k > 0) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) *reinterpret_cast<float4*>(&other[part_k - 1][kMine * ty + i][4 * tx]) = make_float4(acc[i][0].x, acc[i][0].y, acc[i][1].x, acc[i][1].y);
  }
  __syncthreads();
  if (part_k == 0) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      float4 sum = make_float4(acc[i][0].x, acc[i][0].y, acc[i][1].x, acc[i][1].y);
#pragma unroll
      for (int q = 0; q < kParts - 1; ++q) {
        const float4 o = *reinterpret_cast<const float4*>(&other[q][kMine * ty + i][4 * tx]);
        sum.x += o.x; sum.y += o.y; sum.z += o.z; sum.w += o.w;
      }
      *reinterpret_cast<float4*>(&tile[kMine * ty + i][4 * tx]) = sum;
    }
  }
  if (splits > 1) cluster_meet();
  else __syncthreads();

  // This CTA's rows of the tile, four columns a thread.
  const TrainEpilogue& e = g.epi;
  const int rows = kRows / splits, r0 = split * rows;
  auto sums = [&](int r, int c, float* v) {
    if (splits == 1) {
      const float4 f = *reinterpret_cast<const float4*>(&tile[r][c]);
      v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
      return;
    }
    float4 f[kMaxSplit];  // every load is under way before the first is added
#pragma unroll
    for (int s = 0; s < kMaxSplit; ++s) f[s] = s < splits ? remote_quad(&tile[r][c], s) : make_float4(0.f, 0.f, 0.f, 0.f);
    v[0] = v[1] = v[2] = v[3] = 0.f;
#pragma unroll
    for (int s = 0; s < kMaxSplit; ++s) { v[0] += f[s].x; v[1] += f[s].y; v[2] += f[s].z; v[3] += f[s].w; }
  };
  float* const down = pool;  // kHidden: [rows][kCols] of dz
  static_assert(kRows * (kCols + 4) <= kDepth * (kRows + 4 + kCols + 4), "a tile fits the operands' arrays");
  for (int i = threadIdx.x; i < rows * (kNeurons / 4); i += kThreads) {
    const int r = i / (kNeurons / 4), c = i % (kNeurons / 4) * 4, m = m0 + r0 + r, n = n0 + c;
    const int left = m < g.M ? min(4, g.N - n) : 0;
    float v[4];
    sums(r0 + r, c, v);
    if constexpr (EPI == kEpiStore) {
      if (left > 0) put4(e.out[z], m * e.ld_out + n, v, left);
    } else if constexpr (EPI == kEpiGateUp) {
      float u[4], h[4];
      sums(r0 + r, kNeurons + c, u);
      if (left <= 0) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (e.bias && j < left) v[j] += e.bias[n + j];
        h[j] = train_act<false>(e.act, v[j]) * train_act<false>(e.act_up, u[j]);
      }
      if (e.z) {
        put4(e.z, m * e.ld_zu + n, v, left);
        put4(e.u, m * e.ld_zu + n, u, left);
      }
      put4(e.h, m * e.ld_h + n, h, left);
    } else {
      float zv[4], uv[4], h[4], du[4];
      get4(e.z, m * e.ld_zu + n, zv, left);
      get4(e.u, m * e.ld_zu + n, uv, left);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float a, da, b, db;
        train_act_slope<false>(e.act, zv[j], a, da);
        train_act_slope<false>(e.act_up, uv[j], b, db);
        h[j] = a * b;
        du[j] = v[j] * a * db;
        v[j] = v[j] * b * da;
      }
      if (left > 0) {
        if (e.dz) put4(e.dz, m * e.ld_h + n, v, left);
        if (e.du) put4(e.du, m * e.ld_h + n, du, left);
        if (e.h) put4(e.h, m * e.ld_h + n, h, left);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) down[r * kCols + c + j] = j < left ? v[j] : 0.f;
    }
  }
  if (EPI == kEpiHidden && e.db) {
    __syncthreads();
    if (threadIdx.x < kCols && n0 + threadIdx.x < g.N) {
      float sum = 0.f;
      for (int r = 0; r < rows; ++r) sum += down[r * kCols + threadIdx.x];
      e.db[((int64_t)(m0 / kRows) * splits + split) * e.ld_h + n0 + threadIdx.x] = sum;
    }
  }
  if (splits > 1) cluster_meet();  // nobody leaves while its sums may still be read
}

// One column a lane, eight runs of lines a CTA.
__global__ void __launch_bounds__(256) train_column_sums_kernel(const float* partial, int lines, int64_t ld, int N, float* out) {
  __shared__ float run[8][32];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, n = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (n < N) {
    const int first = lines * part / 8, last = lines * (part + 1) / 8;
#pragma unroll 8
    for (int l = first; l < last; ++l) sum += partial[l * ld + n];
  }
  run[part][lane] = sum;
  __syncthreads();
  if (part == 0 && n < N) {
    sum = run[0][lane];
    for (int q = 1; q < 8; ++q) sum += run[q][lane];
    out[n] = sum;
  }
}

// CTAs that share a tile's K: until there are a few for every SM, while each keeps two pieces.
int splits_for(const TrainGemm& g, int rows) {
  const int neurons = g.epilogue == kEpiGateUp ? kCols / 2 : kCols;
  const long long tiles = (long long)((g.M + rows - 1) / rows) * ((g.N + neurons - 1) / neurons) * g.batch;
  const int pieces = (g.epilogue == kEpiGateUp ? 1 : g.parts) * ((g.K + kDepth - 1) / kDepth);
  int s = 1;
  while (s < kMaxSplit && tiles * s < 6 * 148 && pieces >= 2 * s) s *= 2;
  return s;
}

}  // namespace

int train_simt_lines(int M) { return (M + 31) / 32 * kMaxSplit * (M <= kFewRows ? kFewRows / 8 : 1); }

template <int EPI>
static cudaError_t launch_epilogue(const TrainGemm& g, int* lines, cudaStream_t s) {
  const int rows = g.M <= kFewRows ? 8 : 32;
  const int neurons = EPI == kEpiGateUp ? kCols / 2 : kCols, splits = splits_for(g, rows), m_tiles = (g.M + rows - 1) / rows;
  const long long ctas = (long long)splits * ((g.N + neurons - 1) / neurons) * m_tiles * g.batch;
  if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
  *lines = m_tiles * splits;
  return launch_clusters(splits, rows == 8 ? train_simt_kernel<EPI, 8> : train_simt_kernel<EPI, 32>, dim3((unsigned)ctas), dim3(kThreads), 0, s, g, splits);
}

cudaError_t launch_train_simt(const TrainGemm& g, int* lines, cudaStream_t s) {
  return g.epilogue == kEpiStore ? launch_epilogue<kEpiStore>(g, lines, s)
         : g.epilogue == kEpiGateUp ? launch_epilogue<kEpiGateUp>(g, lines, s) : launch_epilogue<kEpiHidden>(g, lines, s);
}

cudaError_t launch_train_column_sums(const float* partial, int lines, int64_t ld, int N, float* out, cudaStream_t s) {
  return launch_pdl(train_column_sums_kernel, dim3((N + 31) / 32), dim3(256), 0, s, partial, lines, ld, N, out);
}

}  // namespace sffn
