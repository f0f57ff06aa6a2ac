// Products of the Newton-Schulz steps on the 5th-generation tensor cores (tcgen05.mma kind::f16, accumulators in tensor memory).
//
// A step is X' = a X + (b P + c P^2) X with P = X X^T on the shorter side: three products, of which P and P^2 are symmetric: their tiles
// at and below the diagonal are computed, and what lies below it is stored twice.
//
// Operands are fp16, not bf16: the matrices are scaled (powers of two; a bound on every one's entries follows from the coefficients), so
// the exponent range is not needed, and eleven bits are eight times as exact at the same rate.  What would be amplified is kept out
// of sixteen bits: singular values far below the largest grow by a in every step, 485 times in five, and with them the rounding of a X.
// So X is held in two terms, hi + lo, and only the products take hi; and Q's diagonal, its largest entries, goes with a X, in fp32.
// (64-bit model, 1344 x 384, error against exact, norm by norm: Gaussian 7.6e-4, of rank 16 1.0e-3, dying singular values 2e-4 to 5e-4; with
// a X from one term rank 16 2.9e-2, with bf16 operands 1.2e-2 and 0.24.)  Where results are wanted in 32 bits, every operand enters in two
// terms: hi hi in runs of eight K blocks, which are added up in registers because the tensor cores truncate when they add onto an
// accumulator, and hi lo + lo hi in an accumulator of their own.
//
// A pair of CTAs (cta_group::2) owns 256 rows; one term: 512 columns, two accumulators, 48 KB a K block of 64 in four stages; two terms: 256
// columns, 64 KB in three.  X is used as it lies: X^T X takes MN-major boxes, X X^T K-major ones.  Epilogues go from tensor memory through
// registers straight to memory, a lane a row, sixteen columns (32 bytes) at a time; what they read is under way one step ahead.
//
// Tiles are dealt to the pairs round robin; what is left for a last, partly idle round is cut along K where that is shorter, and
// muon_join_kernel adds up the pieces in their order and does the epilogue.  Every wait is bounded by a cycle budget; on expiry the status
// word is set, all roles wind down and tensor memory is given back.
#include <cuda_fp16.h>

#include <cmath>

#include "common.cuh"
#include "fused_kernel.cuh"
#include "muon_kernels.cuh"
#include "tcgen05.cuh"

namespace sffn {
namespace {

using namespace tc;

constexpr int kRows = 256;                   // of a pair's tile
constexpr int kDeep = 64;                    // fp16 elements of a 128-byte swizzle row: a K block
constexpr int kBlockBytes = 128 * kDeep * 2; // 128 rows of a K block
constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;            // warps 4-11
constexpr int kRun = 8;                      // two terms: K blocks of a run

template <int TERMS>
struct Form {
  static constexpr int kWide = TERMS == 1 ? 2 : 1;         // accumulators side by side
  static constexpr int kCols = 256 * kWide;
  static constexpr int kStages = TERMS == 1 ? 4 : 3;
  static constexpr int kStageBytes = TERMS == 1 ? 3 * kBlockBytes : 4 * kBlockBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + 1024;
};

struct Maps {
  CUtensorMap a[2], b[2];  // hi, lo
};

struct Params {
  int kind, M, N, K, n;           // n: matrices
  int m_tiles, n_tiles, per, tiles, blocks;
  int whole, split;               // tiles dealt whole; pieces of each of the others
  int a_mn, b_mn;
  float* partial;
  int piece;                      // floats of a piece
  int32_t* status;
  long long budget;
  int drop;                       // test hook: a K block whose rows of A CTA 0 leaves out (-1: none)
  // epilogue
  int tall, first, last;
  float a, b, c;                  // of what is stored: alpha for kGram in c
  const float* factors;           // first step: [n][4]
  float x_scale, acc_scale;       // kApply: of a X, and of the accumulator
  float diag_scale;               // kPoly: from Q as stored to Q
  const uint16_t* in;             // kPoly: P; kApply: X
  uint16_t* out;                  // kGram: P; kPoly: Q; kApply: X'
  int64_t ld, matrix, term;       // of both
  float* diag;
  int S;
  // last step
  int step, out_bf16;
  const float* grad_norm;
  MuonItem item[kMuonBatch];
};

struct Place {
  int batch, m, n;
};
// Where a tile lies.  Symmetric products: tiles that reach the diagonal or lie below it, two rows of tiles by two (by one, with one
// accumulator a tile).  Others: groups of eight tile rows, column by column, so that what runs at one time shares rows and columns in L2.
template <int KIND, int WIDE>
__device__ __forceinline__ Place place_of(const Params& p, int tile) {
  Place at;
  at.batch = tile / p.per;
  tile -= at.batch * p.per;
  if constexpr (KIND != kApply) {
    if constexpr (WIDE == 1) {
      int m = (int)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
      while (m * (m + 1) / 2 > tile) --m;
      while ((m + 1) * (m + 2) / 2 <= tile) ++m;
      at.m = m;
      at.n = tile - m * (m + 1) / 2;
    } else {
      int q = (int)((sqrtf(4.f * tile + 1.f) - 1.f) * 0.5f);
      while (q * (q + 1) > tile) --q;
      while ((q + 1) * (q + 2) <= tile) ++q;
      const int rest = tile - q * (q + 1), two = 2 * q + 1 < p.m_tiles;
      at.m = 2 * q + (two ? rest & 1 : 0);
      at.n = two ? rest >> 1 : rest;
    }
  } else {
    constexpr int kGroup = 8;
    const int group = tile / (kGroup * p.n_tiles), first = group * kGroup, rows = min(kGroup, p.m_tiles - first);
    tile -= first * p.n_tiles;
    at.m = first + tile % rows;
    at.n = tile / rows;
  }
  return at;
}
// Accumulators of a tile that have columns to compute.
template <int KIND, int WIDE>
__device__ __forceinline__ int halves_of(const Params& p, const Place& at) {
  if (WIDE == 1) return 1;
  if (KIND != kApply) return 2 * at.n + 1 <= at.m ? 2 : 1;
  return at.n * 512 + 256 < p.N ? 2 : 1;
}

// A pair's pieces of work in order: pieces of the tiles that are cut, then whole tiles.
struct Item {
  int tile, u0, u1, piece;
};
struct Walk {
  int pairs, next_piece, next;
  __device__ __forceinline__ Walk(int pairs_, int pair) : pairs(pairs_), next_piece(pair), next(pair) {}
  __device__ __forceinline__ bool step(const Params& p, Item& it) {
    const int cut = p.tiles - p.whole;
    if (next_piece < cut * p.split) {
      const int part = next_piece / cut;
      it.tile = p.whole + next_piece - part * cut;
      it.u0 = (int)((long long)p.blocks * part / p.split);
      it.u1 = (int)((long long)p.blocks * (part + 1) / p.split);
      it.piece = next_piece;
      next_piece += pairs;
      return true;
    }
    if (next >= p.whole) return false;
    it.tile = next;
    it.u0 = 0;
    it.u1 = p.blocks;
    it.piece = -1;
    next += pairs;
    return true;
  }
};

// ---- epilogue: sixteen columns from n0 on of the row m = row0 + lane ------------------------------------------------

__device__ __forceinline__ void half8(const uint4& w, float* f) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}
__device__ __forceinline__ uint32_t two_halves(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float rest_of_half(float v) { return v - __half2float(__float2half_rn(v)); }
__device__ __forceinline__ void put16(uint16_t* to, const float* v) {  // 32 bytes
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = two_halves(v[2 * i], v[2 * i + 1]);
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
               "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void get32(const void* from, uint4* w) {  // 32 bytes
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y), "=r"(w[1].z), "=r"(w[1].w)
               : "l"(from)
               : "memory");
}

// What a chunk's epilogue reads, under way while the one before is worked on.
struct Ahead {
  uint4 hi[2], lo[2];
  uint4 w[4];      // last step: the parameter, sixteen fp32 or bf16
  float d;         // the diagonal: lane l has column n0 + l's (tall), or its row's
};
// Whether a row of the caller's can be read and written sixteen columns at a time.
__device__ __forceinline__ bool wide_row(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

template <int KIND, int TERMS>
__device__ __forceinline__ void load_ahead(const Params& p, int batch, int m, int n0, int lane, Ahead& t) {
  if constexpr (KIND == kGram) return;
  const bool row = m < p.M && n0 < p.N;
  if (row) {
    const uint16_t* from = p.in + batch * p.matrix + (int64_t)m * p.ld + n0;
    get32(from, t.hi);
    if (KIND == kApply || TERMS == 2) get32(from + p.term, t.lo);
  }
  if constexpr (KIND == kApply) {
    const float* d = p.diag + (int64_t)batch * p.S;
    t.d = 0.f;
    if (p.tall) {
      if (lane < 16 && n0 + lane < p.N) t.d = d[n0 + lane];
    } else if (m < p.M) {
      t.d = d[m];
    }
    if (p.last && p.step && row && n0 + 16 <= p.N) {
      const MuonItem& it = p.item[batch];
      const int64_t at = (int64_t)m * it.ld_out + n0;
      if (it.master || !p.out_bf16) {
        const float* w = (it.master ? it.master : static_cast<float*>(it.out)) + at;
        if (wide_row(w, 32)) {
          get32(w, t.w);
          get32(w + 8, t.w + 2);
        }
      } else {
        const uint16_t* w = static_cast<uint16_t*>(it.out) + at;
        if (wide_row(w, 32)) get32(w, t.w);
      }
    }
  }
}

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void out_bf16(uint16_t* to, const float* v, int count) {
  if (count == 16 && wide_row(to, 32)) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = two_bf16(v[2 * i], v[2 * i + 1]);
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]),
                 "r"(w[7])
                 : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < count) to[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
  }
}
__device__ __forceinline__ void out_f32(float* to, const float* v, int count) {
  if (count == 16 && wide_row(to, 32)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to + 8 * h), "f"(v[8 * h]), "f"(v[8 * h + 1]), "f"(v[8 * h + 2]),
                   "f"(v[8 * h + 3]), "f"(v[8 * h + 4]), "f"(v[8 * h + 5]), "f"(v[8 * h + 6]), "f"(v[8 * h + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < count) to[i] = v[i];
  }
}

// The caller's sixteen entries: O itself, or p = decay p - rate O.
__device__ __forceinline__ void finish_last(const Params& p, int batch, int m, int n0, float* v, const Ahead& t) {
  const MuonItem& it = p.item[batch];
  const int count = min(16, p.N - n0);
  const int64_t at = (int64_t)m * it.ld_out + n0;
  if (p.step) {
    if (p.grad_norm && !isfinite(*p.grad_norm)) return;
    float w[16];
    const bool f32 = it.master || !p.out_bf16;
    float* const wide = (it.master ? it.master : static_cast<float*>(it.out)) + at;
    uint16_t* const narrow = static_cast<uint16_t*>(it.out) + at;
    const bool had = count == 16 && wide_row(f32 ? static_cast<const void*>(wide) : narrow, 32);
    if (f32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[4 * i] = __uint_as_float(t.w[i].x); w[4 * i + 1] = __uint_as_float(t.w[i].y);
        w[4 * i + 2] = __uint_as_float(t.w[i].z); w[4 * i + 3] = __uint_as_float(t.w[i].w);
      }
    } else {
      Elem<__nv_bfloat16>::unpack(t.w[0], w);
      Elem<__nv_bfloat16>::unpack(t.w[1], w + 8);
    }
    if (!had) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < count) w[i] = f32 ? wide[i] : __uint_as_float((uint32_t)narrow[i] << 16);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf(-it.rate, v[i], it.decay * w[i]);
    if (it.master) out_f32(it.master + at, v, count);
  }
  if (p.out_bf16) out_bf16(static_cast<uint16_t*>(it.out) + at, v, count);
  else out_f32(static_cast<float*>(it.out) + at, v, count);
}

// v: the accumulators of these sixteen columns.  All lanes of a warp come here together.
template <int KIND, int TERMS>
__device__ __forceinline__ void finish(const Params& p, int batch, int row0, int n0, int lane, float* v, const Ahead& t) {
  const int m = row0 + lane;
  const bool row = m < p.M;
  if constexpr (KIND == kApply) {
    const float a = p.first ? p.a * p.factors[4 * batch] : p.a;
    float hi[16], lo[16];
    half8(t.hi[0], hi);
    half8(t.hi[1], hi + 8);
    half8(t.lo[0], lo);
    half8(t.lo[1], lo + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float d = p.tall ? __shfl_sync(0xffffffffu, t.d, i) : t.d;
      v[i] = fmaf((a + d) * p.x_scale, hi[i] + lo[i], v[i] * p.acc_scale);
    }
    if (!row) return;
    if (p.last) {
      finish_last(p, batch, m, n0, v, t);
      return;
    }
  } else {
    float scale = p.c, linear = p.b;
    if (KIND == kPoly && p.first) {
      linear *= p.factors[4 * batch + 1];
      scale *= p.factors[4 * batch + 2];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= scale;
    if constexpr (KIND == kPoly) {
      float f[16];
      half8(t.hi[0], f);
      half8(t.hi[1], f + 8);
      if constexpr (TERMS == 2) {
        float lo[16];
        half8(t.lo[0], lo);
        half8(t.lo[1], lo + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] += lo[i];
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = fmaf(linear, f[i], v[i]);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (n0 + i == m && row) {
          p.diag[(int64_t)batch * p.S + m] = v[i] * p.diag_scale;
          v[i] = 0.f;
        }
    }
  }
  uint16_t* const out = p.out + batch * p.matrix;
  if (row) {
    put16(out + (int64_t)m * p.ld + n0, v);
    if (KIND == kApply || TERMS == 2) {
      float r[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) r[i] = rest_of_half(v[i]);
      put16(out + p.term + (int64_t)m * p.ld + n0, r);
    }
  }
  if constexpr (KIND != kApply) {
    if (row && (n0 >> 5) < (row0 >> 5)) {  // below the diagonal: the same above it
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (n0 + i >= p.N) continue;
        uint16_t* const to = out + (int64_t)(n0 + i) * p.ld + m;
        *to = __half_as_ushort(__float2half_rn(v[i]));
        if (TERMS == 2) to[p.term] = __half_as_ushort(__float2half_rn(rest_of_half(v[i])));
      }
    }
  }
}
// Whether a chunk is there to be computed.
template <int KIND>
__device__ __forceinline__ bool wanted(const Params& p, int row0, int n0) {
  return n0 < p.N && (KIND == kApply || (n0 >> 5) <= (row0 >> 5));
}

__device__ __forceinline__ void put_piece(float* at, const float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at + 8 * h), "f"(v[8 * h]), "f"(v[8 * h + 1]), "f"(v[8 * h + 2]), "f"(v[8 * h + 3]),
                 "f"(v[8 * h + 4]), "f"(v[8 * h + 5]), "f"(v[8 * h + 6]), "f"(v[8 * h + 7])
                 : "memory");
}

__device__ __forceinline__ uint32_t idesc_f16(int m, int n, bool a_mn, bool b_mn) {  // D fp32, A and B fp16
  return (1u << 4) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <int KIND, int TERMS>
__global__ void __launch_bounds__(kThreads, 1) muon_umma_kernel(const __grid_constant__ Params p, const __grid_constant__ Maps maps) {
  using F = Form<TERMS>;
  constexpr int kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(8) uint64_t bars[2 * kStages + 4];
  volatile int* const abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
  const int rank = (int)cluster_rank(), pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full + 8 * b, 1);
      mbar_init(acc_empty + 8 * b, 2 * kEpilogueWarps);
    }
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  cluster_sync();
  fence_after();
  const uint32_t tmem = tmem_slot;
  // a step's last launch writes parameters, which calls of the inference side read before they wait: nothing starts early behind it
  if (!(p.last && p.step && p.whole == p.tiles)) pdl_launch_dependents();
  pdl_wait();

  Walk walk(pairs, pair);
  Item it;
  auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, p.budget)) != 0; };

  if (warp == 0) {
    int s = 0, phase = 0, left_out = blockIdx.x == 0 ? p.drop : -1;
    bool ok = true;
    while (ok && walk.step(p, it)) {
      const Place at = place_of<KIND, F::kWide>(p, it.tile);
      const int m0 = at.m * kRows + rank * 128, n0 = at.n * F::kCols + rank * 128, halves = halves_of<KIND, F::kWide>(p, at);
      for (int u = it.u0; u < it.u1; ++u) {
        ok = wait_all(empty + 8 * s, phase ^ 1);
        if (!ok) break;
        if (elect_one()) {
          const int k0 = u * kDeep;
          const uint32_t bar = map_rank(full + 8 * s, 0), da = ring + s * F::kStageBytes;
          if (rank == 0) mbar_expect_tx(full + 8 * s, 2 * TERMS * (1 + halves) * kBlockBytes);
          const bool leave = left_out-- == 0;
#pragma unroll
          for (int q = 0; q < TERMS; ++q) {
            const uint32_t to = da + q * kBlockBytes;
            if (leave) continue;
            if (p.a_mn) {
              tma_tile_3d(to, &maps.a[q], m0, k0, at.batch, bar);
              tma_tile_3d(to + kBlockBytes / 2, &maps.a[q], m0 + 64, k0, at.batch, bar);
            } else {
              tma_tile_3d(to, &maps.a[q], k0, m0, at.batch, bar);
            }
          }
          for (int h = 0; h < TERMS * halves; ++h) {  // one term: halves of the columns; two: hi and lo
            const uint32_t to = da + (TERMS + h) * kBlockBytes;
            const CUtensorMap* map = &maps.b[TERMS == 2 ? h : 0];
            const int n = TERMS == 2 ? n0 : n0 + 256 * h;
            if (p.b_mn) {
              tma_tile_3d(to, map, n, k0, at.batch, bar);
              tma_tile_3d(to + kBlockBytes / 2, map, n + 64, k0, at.batch, bar);
            } else {
              tma_tile_3d(to, map, k0, n, at.batch, bar);
            }
          }
        }
        __syncwarp();
        if (++s == kStages) { s = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1 && rank == 0) {
    const uint32_t idesc = idesc_f16(kRows, 256, p.a_mn, p.b_mn);
    const uint64_t a0 = p.a_mn ? desc_mn_major(ring, kBlockBytes / 2) : desc_k_major(ring);
    const uint32_t ring_b = ring + TERMS * kBlockBytes;
    const uint64_t b0 = p.b_mn ? desc_mn_major(ring_b, kBlockBytes / 2) : desc_k_major(ring_b);
    const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // sixteen k
    constexpr uint32_t kNext = kBlockBytes >> 4;
    int s = 0, phase = 0, acc_phase[2] = {1, 1};
    auto multiply = [&](int buffer, int ta, int tb, uint32_t more) {  // terms (or halves) ta, tb of a K block
      const uint32_t off = (uint32_t)(s * F::kStageBytes) >> 4;
#pragma unroll
      for (int k = 0; k < kDeep / 16; ++k)
        umma_pair(tmem + buffer * 256, a0 + off + ta * kNext + k * a_step, b0 + off + tb * kNext + k * b_step, idesc, k > 0 ? 1u : more);
    };
    bool ok = true;
    while (ok && walk.step(p, it)) {
      const int halves = halves_of<KIND, F::kWide>(p, place_of<KIND, F::kWide>(p, it.tile));
      for (int u = it.u0; ok && u < it.u1;) {
        const int end = TERMS == 2 ? min(it.u1, u + kRun) : it.u1;
        for (int n = u; n < end; ++n) {
          ok = wait_all(full + 8 * s, phase);
          if (!ok) break;
          if constexpr (TERMS == 1) {
            // the first block waits for the accumulators, half by half
            for (int h = 0; h < halves; ++h) {
              if (n == u) {
                ok = wait_all(acc_empty + 8 * h, h ? acc_phase[1] : acc_phase[0]);
                if (!ok) break;
                if (h) acc_phase[1] ^= 1;
                else acc_phase[0] ^= 1;
              }
              fence_after();
              if (elect_one()) {
                multiply(h, 0, h, n > u);
                if (h == halves - 1) commit_pair(empty + 8 * s);
                if (n == end - 1) commit_pair(acc_full + 8 * h);
              }
              __syncwarp();
            }
          } else {
            // hi hi waits for the run before to be read, hi lo + lo hi for the tile before
            if (n == u) {
              ok = wait_all(acc_empty, acc_phase[0]);
              acc_phase[0] ^= 1;
              if (ok && u == it.u0) {
                ok = wait_all(acc_empty + 8, acc_phase[1]);
                acc_phase[1] ^= 1;
              }
              if (!ok) break;
            }
            fence_after();
            if (elect_one()) {
              multiply(1, 0, 1, n > it.u0);
              multiply(1, 1, 0, 1);
              multiply(0, 0, 0, n > u);
              commit_pair(empty + 8 * s);
              if (n == end - 1) commit_pair(acc_full);
            }
            __syncwarp();
          }
          if (!ok) break;
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
        u = end;
      }
    }
  } else if (warp >= 4) {
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    constexpr int kChunks = 8;  // of sixteen columns, of a warp and accumulator
    const uint32_t empty0 = map_rank(acc_empty, 0);
    int full_phase[2] = {0, 0};
    bool ok = true;
    auto wait_full = [&](int buffer) {
      const bool there = wait_all(acc_full + 8 * buffer, buffer ? full_phase[1] : full_phase[0]);
      if (buffer) full_phase[1] ^= 1;
      else full_phase[0] ^= 1;
      fence_after();
      return there;
    };
    auto give_back = [&](int buffer) {
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty0 + 8 * buffer);
    };
    while (ok && walk.step(p, it)) {
      const Place at = place_of<KIND, F::kWide>(p, it.tile);
      const int row0 = at.m * kRows + rank * 128 + 32 * quad;  // this warp's first row
      const bool rows = row0 < p.M;                            // has any: the others only keep step
      float* const piece = it.piece < 0 ? nullptr : p.partial + (size_t)it.piece * p.piece + (size_t)(rank * 128 + 32 * quad + lane) * F::kCols;
      const int halves = halves_of<KIND, F::kWide>(p, at);
      if constexpr (TERMS == 2) {
        float acc[16 * kChunks];
#pragma unroll
        for (int i = 0; i < 16 * kChunks; ++i) acc[i] = 0.f;
#pragma unroll 1
        for (int u = it.u0; u < it.u1; u += kRun) {
          ok = wait_full(0);
          if (!ok) break;
          if (rows) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              float v[16];
              tmem_ld16(tmem + lanes + 128 * half + 16 * c, v);
              tmem_arrived(v);
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[16 * c + i] += v[i];
            }
          }
          if (u + kRun < it.u1) give_back(0);
        }
        if (!ok) break;
        // the last run's commit stands for all products of the tile: the small ones are there too.  The sums go back to where the
        // runs were, as a loop over chunks needs.
        if (rows) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            float v[16];
            tmem_ld16(tmem + 256 + lanes + 128 * half + 16 * c, v);
            tmem_arrived(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[16 * c + i] += v[i];
            tmem_st16(tmem + lanes + 128 * half + 16 * c, acc + 16 * c);
          }
          tmem_stored();
        }
        give_back(1);
      }
      for (int h = 0; h < halves; ++h) {
        const int n_base = at.n * F::kCols + 256 * h + 128 * half;
        Ahead next;
        if (rows && !piece && wanted<KIND>(p, row0, n_base)) load_ahead<KIND, TERMS>(p, at.batch, row0 + lane, n_base, lane, next);
        if constexpr (TERMS == 1) {
          ok = wait_full(h);
          if (!ok) break;
        }
        const uint32_t acc = tmem + lanes + h * 256 + 128 * half;
        if (rows && piece) {
#pragma unroll 2
          for (int c = 0; c < kChunks; ++c) {
            float v[16];
            tmem_ld16(acc + 16 * c, v);
            tmem_arrived(v);
            put_piece(piece + 256 * h + 128 * half + 16 * c, v);
          }
        } else if (rows) {
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            const int n0 = n_base + 16 * c;
            if (!wanted<KIND>(p, row0, n0)) break;  // nor is any further one
            const Ahead now = next;
            float v[16];
            tmem_ld16(acc + 16 * c, v);
            if (c + 1 < kChunks && wanted<KIND>(p, row0, n0 + 16)) load_ahead<KIND, TERMS>(p, at.batch, row0 + lane, n0 + 16, lane, next);
            tmem_arrived(v);
            finish<KIND, TERMS>(p, at.batch, row0, n0, lane, v, now);
          }
        }
        give_back(h);
      }
    }
  }

  // Everybody meets, then the allocating warps free tensor memory.  (After a wait that ran out, copies and MMAs may still be in
  // flight: they end within microseconds, and shared memory and tensor memory are only given back after that.)
  if (*abort_flag)
    for (int i = 0; i < 50; ++i) __nanosleep(1000);
  fence_before();
  cluster_sync();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// The tiles that were cut along K: a warp has 32 rows x 16 columns, adds up their pieces in the order of K and does the epilogue.
constexpr int kJoinWarps = 4;
template <int KIND, int TERMS>
__global__ void __launch_bounds__(32 * kJoinWarps) muon_join_kernel(const __grid_constant__ Params p) {
  using F = Form<TERMS>;
  const int lane = threadIdx.x & 31, number = blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (!(p.last && p.step)) pdl_launch_dependents();
  pdl_wait();
  constexpr int kAcross = F::kCols / 16, kPer = kAcross * (kRows / 32);
  const int t = number / kPer, in = number % kPer, r0 = in / kAcross * 32, c0 = in % kAcross * 16;
  if (t >= p.tiles - p.whole) return;
  const Place at = place_of<KIND, F::kWide>(p, p.whole + t);
  const int row0 = at.m * kRows + r0, n0 = at.n * F::kCols + c0;
  if (row0 >= p.M || !wanted<KIND>(p, row0, n0)) return;
  Ahead now;
  load_ahead<KIND, TERMS>(p, at.batch, row0 + lane, n0, lane, now);
  float v[16] = {};
  const float* from = p.partial + (size_t)t * p.piece + (size_t)(r0 + lane) * F::kCols + c0;
  const size_t next = (size_t)(p.tiles - p.whole) * p.piece;
#pragma unroll 4
  for (int q = 0; q < p.split; ++q, from += next) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = __ldcg(reinterpret_cast<const float4*>(from) + i);
      v[4 * i] += f.x; v[4 * i + 1] += f.y; v[4 * i + 2] += f.z; v[4 * i + 3] += f.w;
    }
  }
  finish<KIND, TERMS>(p, at.batch, row0, n0, lane, v, now);
}

// ---- host ------------------------------------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    cudaDriverEntryPointQueryResult q;
    void* ptr = nullptr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

// `n` fp16 matrices [rows, width] in boxes of 64 elements x `box` rows, 128-byte swizzle.
bool make_map(CUtensorMap* m, const void* base, int64_t width, int64_t rows, int64_t ld, int n, int64_t matrix, int box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)n};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)matrix * 2};
  const cuuint32_t boxes[3] = {(cuuint32_t)kDeep, (cuuint32_t)box, 1};
  const cuuint32_t steps[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of a product of one matrix.
int tiles_of(int kind, int wide, int M, int N, int* m_tiles, int* n_tiles) {
  const int m = (M + kRows - 1) / kRows, n = (N + 256 * wide - 1) / (256 * wide);
  if (m_tiles) *m_tiles = m;
  if (n_tiles) *n_tiles = n;
  if (kind == kApply) return m * n;
  if (wide == 1) return m * (m + 1) / 2;
  return m / 2 * (m / 2 + 1) + (m & 1 ? m / 2 + 1 : 0);
}

// Whole rounds of tiles, then the rest: whole too, or cut along K into equal pieces, dealt in rounds of their own.  What is shortest, counted in
// K blocks: a piece's rows are written to the workspace, and a kernel of its own joins the pieces.
int plan(Params& p, int wide, int terms, int pairs) {
  const int rest = p.tiles % pairs;
  p.whole = p.tiles;
  p.split = 1;
  if (rest > 0) {
    const double products = terms == 2 ? 3 : 1, piece = 1.0 + 8.0 * wide;
    double best = p.blocks * products;
    for (int split = 2; split <= p.blocks && rest * split <= kMuonPieces; ++split) {
      const int rounds = (rest * split + pairs - 1) / pairs;
      const double time = rounds * (std::ceil((double)p.blocks / split) * products + piece) + 5.0 + 0.5 * split;
      if (time < best) {
        best = time;
        p.split = split;
      }
    }
    if (p.split > 1) p.whole = p.tiles - rest;
  }
  const int pieces = (p.tiles - p.whole) * p.split, most = p.whole > pieces ? p.whole : pieces;
  return most < pairs ? most : pairs;
}

template <int KIND, int TERMS>
cudaError_t launch(const MuonBatch& b, Params& p, const Maps& maps, int sm_count, cudaStream_t s) {
  using F = Form<TERMS>;
  const int per = tiles_of(KIND, F::kWide, p.M, p.N, &p.m_tiles, &p.n_tiles);
  p.per = per;
  p.tiles = per * b.n;
  p.blocks = (p.K + kDeep - 1) / kDeep;
  p.piece = kRows * F::kCols;
  const int most = sm_count / 2 < kMuonPairs ? sm_count / 2 : kMuonPairs;
  const int pairs = plan(p, F::kWide, TERMS, most);
  static unsigned long long configured = 0;
  cudaError_t e = allow_dynamic_smem(muon_umma_kernel<KIND, TERMS>, F::kSmemBytes, configured);
  if (e != cudaSuccess) return e;
  e = launch_clusters(2, muon_umma_kernel<KIND, TERMS>, dim3(2 * pairs), dim3(kThreads), F::kSmemBytes, s, p, maps);
  if (e != cudaSuccess || p.whole == p.tiles) return e;
  const int warps = (p.tiles - p.whole) * (F::kCols / 16) * (kRows / 32);
  return launch_pdl(muon_join_kernel<KIND, TERMS>, dim3((warps + kJoinWarps - 1) / kJoinWarps), dim3(32 * kJoinWarps), 0, s, p);
}

}  // namespace

size_t muon_partial_floats(int S, int R, int C, int n, int terms) {
  size_t most = 0;
  const int wide = terms == 1 ? 2 : 1;
  for (int kind : {kGram, kPoly, kApply}) {
    const long long K = kind == kGram ? (R > C ? R : C) : S, blocks = (K + kDeep - 1) / kDeep;
    const long long tiles = (long long)tiles_of(kind, wide, kind == kApply ? R : S, kind == kApply ? C : S, nullptr, nullptr) * n;
    const long long pieces = blocks < 2 ? 0 : tiles < kMuonPieces && tiles * blocks < kMuonPieces ? tiles * blocks : kMuonPieces;
    const size_t floats = (size_t)pieces * kRows * 256 * wide;
    if (floats > most) most = floats;
  }
  return most;
}

cudaError_t launch_muon_product(const MuonBatch& b, const MuonProduct& q, int sm_count, cudaStream_t s) {
  Params p{};
  p.kind = q.kind;
  p.n = b.n;
  p.S = b.S;
  p.M = q.kind == kApply ? b.R : b.S;
  p.N = q.kind == kApply ? b.C : b.S;
  p.K = q.kind == kGram ? b.L : b.S;
  p.partial = b.partial;
  p.status = b.status;
  p.budget = fused_test_knobs().wait_cycles;
  p.drop = fused_test_knobs().drop_stage;
  p.tall = b.tall;
  p.first = q.first;
  p.last = q.last;
  p.factors = b.first;
  p.diag = b.diag;
  const uint16_t *const X = b.x[q.from];
  uint16_t* const Y = b.x[q.from ^ 1];
  auto two = [](int e) { return (float)std::ldexp(1.0, e); };
  Maps maps;
  bool fine = true;
  for (int t = 0; t < b.terms && fine; ++t) {
    const uint16_t *const x = X + t * b.x_term, *const P = b.P + t * b.p_term, *const Q = b.Q + t * b.p_term;
    if (q.kind == kGram) {  // rows of X are k where it is tall
      fine = make_map(&maps.a[t], x, b.C, b.R, b.ld_x, b.n, b.x_matrix, b.tall ? 64 : 128);
      maps.b[t] = maps.a[t];
      p.a_mn = p.b_mn = b.tall;
    } else if (q.kind == kPoly) {
      fine = make_map(&maps.a[t], P, b.S, b.S, b.ld_p, b.n, b.p_matrix, 128);
      maps.b[t] = maps.a[t];
    } else if (b.tall) {
      fine = make_map(&maps.a[t], x, b.C, b.R, b.ld_x, b.n, b.x_matrix, 128) && make_map(&maps.b[t], Q, b.S, b.S, b.ld_p, b.n, b.p_matrix, 128);
    } else {
      fine = make_map(&maps.a[t], Q, b.S, b.S, b.ld_p, b.n, b.p_matrix, 128) && make_map(&maps.b[t], x, b.C, b.R, b.ld_x, b.n, b.x_matrix, 64);
      p.b_mn = 1;
    }
  }
  if (!fine) return cudaErrorInvalidValue;
  if (b.terms == 1) maps.a[1] = maps.a[0], maps.b[1] = maps.b[0];
  if (q.kind == kGram) {
    p.c = two(q.ep - 2 * q.ex);
    p.out = b.P;
    p.ld = b.ld_p; p.matrix = b.p_matrix; p.term = b.p_term;
    return b.terms == 1 ? launch<kGram, 1>(b, p, maps, sm_count, s) : launch<kGram, 2>(b, p, maps, sm_count, s);
  }
  if (q.kind == kPoly) {
    p.b = q.b * two(q.eq - q.ep);
    p.c = q.c * two(q.eq - 2 * q.ep);
    p.diag_scale = two(-q.eq);
    p.in = b.P;
    p.out = b.Q;
    p.ld = b.ld_p; p.matrix = b.p_matrix; p.term = b.p_term;
    return b.terms == 1 ? launch<kPoly, 1>(b, p, maps, sm_count, s) : launch<kPoly, 2>(b, p, maps, sm_count, s);
  }
  p.a = q.a;
  p.x_scale = two((q.last ? 0 : q.ey) - q.ex);
  p.acc_scale = two((q.last ? 0 : q.ey) - q.ex - q.eq);
  p.in = X;
  p.out = Y;
  p.ld = b.ld_x; p.matrix = b.x_matrix; p.term = b.x_term;
  p.step = b.step;
  p.out_bf16 = b.out_bf16;
  p.grad_norm = b.grad_norm;
  if (q.last)
    for (int i = 0; i < b.n; ++i) p.item[i] = b.item[i];
  return b.terms == 1 ? launch<kApply, 1>(b, p, maps, sm_count, s) : launch<kApply, 2>(b, p, maps, sm_count, s);
}

}  // namespace sffn
