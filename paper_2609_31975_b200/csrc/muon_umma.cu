// Products of the Newton-Schulz steps on the 5th-generation tensor cores (tcgen05.mma kind::f16, accumulators in tensor memory).
//
// A step is X' = a X + (b A + c A^2) X with A = X X^T on the shorter side S.  Steps in company go on from A instead of X:
//     B = b A + c A^2,   D = a A + A B,   A' = a D + D B  (= X' X'^T),   B' = b' A' + c' A'^2,   R = a B' + a' B + B B',   X'' = a a' X + R X
// one product with X for all of them and one Gram matrix, for four products of S x S a step.  All of these are polynomials of A, so
// symmetric, and each is one form m M + n N + k M N: tiles at and below the diagonal are computed, and what lies below it is stored
// twice.  (A' = a^2 A + 2 a A B + A B B would lose four bits: its terms are 20 times as large as what is left of them.)
//
// Operands are fp16, not bf16: matrices are scaled (powers of two; a bound on every one's entries follows from the coefficients), so
// the exponent range is not needed, and eleven bits are eight times as exact at the same rate.  What would be amplified is kept out
// of sixteen bits: singular values far below the largest grow by a in every step, 485 times in five, and with them the rounding of a X.
// So X is held in two terms, hi + lo, and only the products take hi.  And every symmetric matrix is held as its diagonal, in fp32, and the
// rest: diagonals are the largest entries by far, and what they contribute to a product is added in the epilogue.
// What the diagonal of R contributes to R X takes both terms of X only in the last steps.  In R hi all is within the column space of R,
// but with both terms for the diagonal alone what is wrong is (R - diag) lo, 2^-12 diag of it outside of every singular vector of X, to be
// multiplied by a in each step to come: fine for X of full rank (five times as exact, R is near its diagonal then), but of rank 1 a matrix of
// 4 x 19 came out 3.3e-2 off.  So: both where what is to come multiplies it by four at most (1.5e-3).
// (64-bit model, 1344 x 384, error against exact, norm by norm, steps one by one / in pairs: Gaussian 6e-4 / 5e-4, of rank 16 1.2e-3 / 2.2e-3,
// singular values dying away 3e-4 to 5e-4 / 6e-4 to 8e-4, half of them small 2e-3 / 3.6e-3; with a X from one term rank 16 2.9e-2, with bf16 operands 1.2e-2 and 0.24.)
// Where results are wanted in 32 bits, every operand enters in two terms: hi hi in runs of eight K blocks, which are added up in registers
// because the tensor cores truncate when they add onto an accumulator, and hi lo + lo hi in an accumulator of their own.
//
// A pair of CTAs (cta_group::2) owns 256 rows; one term: 512 columns, two accumulators, 48 KB a K block of 64 in four stages, and eight
// epilogue warps for each accumulator, as both hold the next tile up; two terms: 256 columns, 64 KB in three stages, eight epilogue warps
// that add up the runs and finish the tile from their registers under the next one.  X is used as it lies: X^T X takes MN-major boxes,
// X X^T K-major ones.  Epilogues go from tensor memory through registers straight to memory, a lane a row, sixteen columns (32 bytes)
// at a time.
//
// Tiles are dealt to the pairs round robin; what is left for a last, partly idle round is cut along K where that is shorter, and
// muon_join_kernel adds up the pieces in their order and does the epilogue.  Every wait is bounded by a cycle budget; on expiry the status
// word is set, all roles wind down and tensor memory is given back.
//
// Bound by the tensor cores at the power limit (1.42 PFLOP/s over seconds), and, in one term, by the epilogue of X' (half a megabyte an SM a tile).
// 14336 x 4096, one term: Gram matrix 173 us (1.39 PFLOP/s), a form 70 (0.98), X' 408 and 10 for its join (1.15), the last one 384.
// 14230 x 3840, two terms, three products: Gram matrix 490 and 21 us (1.23 PFLOP/s over both), a form 160 and 23 (0.93), X' 942 and 10 (1.32).
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "fused_kernel.cuh"
#include "muon_kernels.cuh"
#include "tcgen05.cuh"

namespace sffn {
namespace {

using namespace tc;

constexpr int kDeep = 64;                    // fp16 elements of a 128-byte swizzle row: a K block
constexpr int kBlockBytes = 128 * kDeep * 2; // 128 rows of a K block
constexpr int kRun = 8;                      // two terms: K blocks of a run

// Pairs' tiles: 256 rows, 512 columns of one term, 256 of two.
template <int TERMS>
struct Form {
  static constexpr int kRows = 256;
  static constexpr int kWide = TERMS == 1 ? 2 : 1;                    // accumulators side by side, of 256 columns
  static constexpr int kCols = 256 * kWide;
  static constexpr int kStages = TERMS == 1 ? 4 : 3;
  static constexpr int kStageBytes = TERMS * (1 + kWide) * kBlockBytes;
  static constexpr int kSmemBytes = kStages * kStageBytes + 1024;
  static constexpr int kWarps = 8;                                   // epilogue warps of an accumulator
  static constexpr int kThreads = 128 + 32 * kWarps * kWide;
};
// Small tiles: a CTA each, two at a time on an SM.
template <int TERMS>
struct Small {
  static constexpr int kRows = 128, kCols = 64;
  static constexpr int kBBytes = kCols * kDeep * 2;
  static constexpr int kStages = 8 / TERMS;                          // half of them where two CTAs share an SM
  static constexpr int kStageBytes = TERMS * (kBlockBytes + kBBytes);
  static constexpr int smem_bytes(int stages) { return stages * kStageBytes + 1024; }
  static constexpr int kRuns = 3;                                    // two terms: runs that have an accumulator
  static constexpr int kTmem = TERMS == 1 ? kCols : (kRuns + 1) * kCols;
  static constexpr int kMostBlocks = TERMS == 1 ? 1 << 20 : kRuns * kRun;  // K blocks of a piece
};

struct Maps {
  CUtensorMap a[2], b[2];  // hi, lo
};

struct Params {
  int M, N, K;
  int m_tiles, n_tiles, per, tiles, blocks;
  int whole, split;               // tiles dealt whole; pieces of each of the others
  int stages;                     // small tiles: of the ring
  int together;                   // small tiles: the pieces of a tile are a cluster, which joins them itself
  int a_mn, b_mn;
  float* partial;
  int piece;                      // floats of a piece
  int32_t* status;
  long long budget;
  int drop;                       // test hook: a K block whose rows of A CTA 0 leaves out (-1: none)
  // epilogue
  int tall, first;
  const float* factors;           // first step: [n][4], powers of g: 1, 2, 3, 5
  int S;
  uint16_t* out;                  // symmetric: the result; kApply: X'
  float* out_diag;
  int64_t ld, matrix, term;       // of X, or of the symmetric matrices
  // symmetric: off the diagonal out = (m + k_m d_N[j]) M + (n + k_n d_M[i]) N + k acc (coefficients as values are stored)
  const uint16_t *M_, *N_;        // N NULL where it is M
  const float *M_diag, *N_diag;
  float m, nn, k_m, k_n, k;
  float dm, dn, dk, dacc;         // the diagonal (as it is): dm d_M + dn d_N + dk (d_M d_N + dacc acc)
  int fm, fn, fk;                 // first step: which factor the terms in m, n, k take (-1: none)
  // kApply, kLast: X' = x_scale (q X + d X) + acc_scale acc, the second X without its second term unless `both` (1 or 0)
  const uint16_t* X;
  const float* diag;
  float q, x_scale, acc_scale, both;
  int fq;
  // kLast
  int step, out_bf16;
  const float* grad_norm;
  MuonItem item[kMuonBatch];
};

struct Place {
  int batch, m, n;
};
// Where a tile lies.  Symmetric products: tiles that reach the diagonal or lie below it, two rows of tiles by two (by one, with one
// accumulator a tile).  Others: groups of eight tile rows, column by column, so that what runs at one time shares rows and columns in L2.
template <int KIND, typename FORM>
__device__ __forceinline__ Place place_of(const Params& p, int tile) {
  Place at;
  at.batch = tile / p.per;
  tile -= at.batch * p.per;
  if constexpr (symmetric(KIND)) {
    if constexpr (FORM::kCols <= FORM::kRows) {  // row m: its kRows / kCols (m + 1) tiles
      constexpr int kEach = FORM::kRows / FORM::kCols;
      int m = (int)((sqrtf(8.f / kEach * tile + 1.f) - 1.f) * 0.5f);
      while (kEach * (m * (m + 1) / 2) > tile) --m;
      while (kEach * ((m + 1) * (m + 2) / 2) <= tile) ++m;
      at.m = m;
      at.n = tile - kEach * (m * (m + 1) / 2);
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
// Accumulators of a pair's tile that have columns to compute.
template <int KIND, int WIDE>
__device__ __forceinline__ int halves_of(const Params& p, const Place& at) {
  if (WIDE == 1) return 1;
  if (symmetric(KIND)) return 2 * at.n + 1 <= at.m ? 2 : 1;
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

// Two fp16 in a word, and sixteen of them in two vectors.
__device__ __forceinline__ uint32_t two_halves(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 from_halves(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
struct Sixteen {
  uint32_t w[8];
  __device__ __forceinline__ void load(const uint16_t* from) {  // 32 bytes
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(from)
                 : "memory");
  }
  __device__ __forceinline__ void store(uint16_t* to) const {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  }
  __device__ __forceinline__ void pack(const float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = two_halves(v[2 * i], v[2 * i + 1]);
  }
  // v - what this holds
  __device__ __forceinline__ void rest(const float* v, float* r) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = from_halves(w[i]);
      r[2 * i] = v[2 * i] - f.x;
      r[2 * i + 1] = v[2 * i + 1] - f.y;
    }
  }
};
// Sixteen numbers of a vector, from n0 on; past its end anything.  (All lanes read the same: the diagonal is padded to a multiple of 16.)
__device__ __forceinline__ void columns16(const float* from, float* d) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 f = __ldcg(reinterpret_cast<const float4*>(from) + i);
    d[4 * i] = f.x; d[4 * i + 1] = f.y; d[4 * i + 2] = f.z; d[4 * i + 3] = f.w;
  }
}
__device__ __forceinline__ int64_t diag_ld(int S) { return (S + 15) / 16 * 16; }
__device__ __forceinline__ float factor(const Params& p, int batch, int which) { return p.first && which >= 0 ? p.factors[4 * batch + which] : 1.f; }

// What all chunks of a warp's row share.
template <int KIND>
struct Shared {
  float d, d_n, f_m, f_n, f_k;  // this row's diagonal (kForm: of M, and of N; X M: none), and the first step's factors
  __device__ __forceinline__ Shared(const Params& p, int batch, int m) : d(0.f), d_n(0.f), f_m(1.f), f_n(1.f), f_k(1.f) {
    const bool row = m < p.M;
    if constexpr (KIND == kForm) {
      if (row) {
        d = __ldcg(p.M_diag + batch * diag_ld(p.S) + m);
        d_n = __ldcg(p.N_diag + batch * diag_ld(p.S) + m);
      }
      if (p.first) {
        f_m = factor(p, batch, p.fm);
        f_n = factor(p, batch, p.fn);
        f_k = factor(p, batch, p.fk);
      }
    } else if constexpr (!symmetric(KIND)) {
      if (row && !p.tall) d = __ldcg(p.diag + batch * diag_ld(p.S) + m);
      f_k = p.q * factor(p, batch, p.fq);
    }
  }
};
// A row's lines on their way into L2: `bytes` from n0's column on.
__device__ __forceinline__ void prefetch_row(const char* from, int bytes) {
  for (int i = 0; i < bytes; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(from + i));
}
// What a warp's epilogue of a tile will read that its products do not: under way while they are computed.
template <int KIND, int COLUMNS>
__device__ __forceinline__ void prefetch(const Params& p, int batch, int m, int n0) {
  if (symmetric(KIND) || m >= p.M || n0 >= p.N) return;  // (symmetric: operands of these products)
  const int64_t at = batch * p.matrix + (int64_t)m * p.ld + n0;
  const int columns = min(COLUMNS, p.N - n0);
  prefetch_row(reinterpret_cast<const char*>(p.X + at), 2 * columns);
  prefetch_row(reinterpret_cast<const char*>(p.X + at + p.term), 2 * columns);
  if (KIND == kLast && p.step) {
    const MuonItem& it = p.item[batch];
    const int64_t to = (int64_t)m * it.ld_out + n0;
    if (it.master) prefetch_row(reinterpret_cast<const char*>(it.master + to), 4 * columns);
    else prefetch_row(static_cast<const char*>(it.out) + to * (p.out_bf16 ? 2 : 4), (p.out_bf16 ? 2 : 4) * columns);
  }
}

// What a chunk's epilogue reads of the matrices in sixteen bits.
template <int KIND, int TERMS>
struct Ahead {
  static constexpr int kTiles = KIND == kForm ? 2 * TERMS : symmetric(KIND) ? 1 : 2;
  Sixteen t[kTiles];
  __device__ __forceinline__ void load(const Params& p, int batch, int m, int n0) {
    if (KIND == kGram || m >= p.M || n0 >= p.N) return;
    const int64_t at = batch * p.matrix + (int64_t)m * p.ld + n0;
    if constexpr (KIND == kForm) {
#pragma unroll
      for (int q = 0; q < TERMS; ++q) {
        t[q].load(p.M_ + at + q * p.term);
        if (p.N_) t[TERMS + q].load(p.N_ + at + q * p.term);
      }
    } else {
      t[0].load(p.X + at);
      t[1].load(p.X + at + p.term);
    }
  }
};

// Whether a row of the caller's can be read and written sixteen columns at a time.
__device__ __forceinline__ bool wide_row(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void row_in(const float* from, float* v, int count) {
  if (count == 16 && wide_row(from)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=f"(v[8 * h]), "=f"(v[8 * h + 1]), "=f"(v[8 * h + 2]), "=f"(v[8 * h + 3]), "=f"(v[8 * h + 4]), "=f"(v[8 * h + 5]), "=f"(v[8 * h + 6]),
                     "=f"(v[8 * h + 7])
                   : "l"(from + 8 * h)
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = i < count ? from[i] : 0.f;
  }
}
__device__ __forceinline__ void row_in(const uint16_t* from, float* v, int count) {  // bf16
  if (count == 16 && wide_row(from)) {
    Sixteen t;
    t.load(from);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[2 * i] = __uint_as_float(t.w[i] << 16);
      v[2 * i + 1] = __uint_as_float(t.w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = i < count ? __uint_as_float((uint32_t)from[i] << 16) : 0.f;
  }
}
__device__ __forceinline__ void row_out(uint16_t* to, const float* v, int count) {  // bf16
  if (count == 16 && wide_row(to)) {
    Sixteen t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.w[i] = two_bf16(v[2 * i], v[2 * i + 1]);
    t.store(to);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < count) to[i] = __bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
  }
}
__device__ __forceinline__ void row_out(float* to, const float* v, int count) {
  if (count == 16 && wide_row(to)) {
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
__device__ __forceinline__ void finish_last(const Params& p, int batch, int m, int n0, float* v) {
  const MuonItem& it = p.item[batch];
  const int count = min(16, p.N - n0);
  const int64_t at = (int64_t)m * it.ld_out + n0;
  if (p.step) {
    if (p.grad_norm && !isfinite(*p.grad_norm)) return;
    float w[16];
    if (it.master) row_in(it.master + at, w, count);
    else if (p.out_bf16) row_in(static_cast<const uint16_t*>(it.out) + at, w, count);
    else row_in(static_cast<const float*>(it.out) + at, w, count);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf(-it.rate, v[i], it.decay * w[i]);
    if (it.master) row_out(it.master + at, v, count);
  }
  if (p.out_bf16) row_out(static_cast<uint16_t*>(it.out) + at, v, count);
  else row_out(static_cast<float*>(it.out) + at, v, count);
}

// Sixteen entries of row m, columns n0 and on, once more where they mirror: rows n0 + i, column m.  Lanes in pairs put two rows' entries of a
// column together.  All lanes of a warp come here.
__device__ __forceinline__ void mirror(const Params& p, uint16_t* out, int m, int n0, int lane, const Sixteen& t) {
  const bool odd = lane & 1, two = (m | 1) < p.M, one = m < p.M;  // (of a last, single row its lane stores both columns alone)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, t.w[i], 1);
    const int n = n0 + 2 * i + odd;
    if (two) {
      if (n < p.N) *reinterpret_cast<uint32_t*>(out + (int64_t)n * p.ld + (m & ~1)) = odd ? __byte_perm(other, t.w[i], 0x7632) : __byte_perm(t.w[i], other, 0x5410);
    } else if (one) {
      if (n < p.N) out[(int64_t)n * p.ld + m] = (uint16_t)t.w[i];
      if (n + 1 < p.N) out[(int64_t)(n + 1) * p.ld + m] = (uint16_t)(t.w[i] >> 16);
    }
  }
}

// What the result has besides the accumulators, of sixteen columns.
template <int KIND, int TERMS>
__device__ __forceinline__ void beside(const Params& p, const Shared<KIND>& all, int batch, int n0, const Ahead<KIND, TERMS>& a, float* v) {
  if constexpr (KIND == kForm) {
    // M = N: their entry once, times m + k (d_M[i] + d_M[j])
    const float by_row = p.k_n * all.f_k * all.d, each = p.k_m * all.f_k, mm = p.N_ ? p.m * all.f_m : p.m * all.f_m + by_row, nn = p.nn * all.f_n + by_row;
    float d[16];
    columns16(p.N_diag + batch * diag_ld(p.S) + n0, d);
#pragma unroll
    for (int i = 0; i < 16; ++i) d[i] = fmaf(each, d[i], mm);
#pragma unroll
    for (int q = 0; q < TERMS; ++q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = from_halves(a.t[q].w[i]);
        v[2 * i] = q ? fmaf(d[2 * i], f.x, v[2 * i]) : d[2 * i] * f.x;
        v[2 * i + 1] = q ? fmaf(d[2 * i + 1], f.y, v[2 * i + 1]) : d[2 * i + 1] * f.y;
      }
      if (p.N_) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = from_halves(a.t[TERMS + q].w[i]);
          v[2 * i] = fmaf(nn, f.x, v[2 * i]);
          v[2 * i + 1] = fmaf(nn, f.y, v[2 * i + 1]);
        }
      }
    }
  } else if constexpr (!symmetric(KIND)) {
    const float q = all.f_k * p.x_scale;
    float d[16];
    if (p.tall) {
      columns16(p.diag + batch * diag_ld(p.S) + n0, d);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) d[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 hi = from_halves(a.t[0].w[i]), lo = from_halves(a.t[1].w[i]);
      v[2 * i] = fmaf((all.d + d[2 * i]) * p.x_scale, fmaf(p.both, lo.x, hi.x), q * (hi.x + lo.x));
      v[2 * i + 1] = fmaf((all.d + d[2 * i + 1]) * p.x_scale, fmaf(p.both, lo.y, hi.y), q * (hi.y + lo.y));
    }
  }
}

// acc: the accumulators of these sixteen columns, more: what is beside them.  All lanes of a warp come here together.
template <int KIND, int TERMS>
__device__ __forceinline__ void finish(const Params& p, const Shared<KIND>& all, int batch, int row0, int n0, int lane, const float* acc, const float* more) {
  const int m = row0 + lane;
  const bool row = m < p.M;
  float v[16];
  if constexpr (!symmetric(KIND)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = fmaf(acc[i], p.acc_scale, more[i]);
    if (!row) return;
    if constexpr (KIND == kLast) {
      finish_last(p, batch, m, n0, v);
    } else {
      uint16_t* const out = p.out + batch * p.matrix + (int64_t)m * p.ld + n0;
      Sixteen t;
      float r[16];
      t.pack(v);
      t.rest(v, r);
      t.store(out);
      t.pack(r);
      t.store(out + p.term);
    }
  } else {
    const float scale = p.k * all.f_k;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = KIND == kGram ? acc[i] * scale : fmaf(acc[i], scale, more[i]);
    if ((n0 >> 5) == (row0 >> 5)) {  // the diagonal goes apart
      float own = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (n0 + i == m) {
          own = acc[i];
          v[i] = 0.f;
        }
      if (row && m >= n0 && m < n0 + 16) {
        const int64_t at = batch * diag_ld(p.S) + m;
        if constexpr (KIND == kGram) {
          p.out_diag[at] = own * p.dacc;
        } else {
          p.out_diag[at] = p.dm * all.f_m * all.d + p.dn * all.f_n * all.d_n + p.dk * all.f_k * fmaf(own, p.dacc, all.d * all.d_n);
        }
      }
    }
    uint16_t* const out = p.out + batch * p.matrix;
    const bool twice = (n0 >> 5) < (row0 >> 5);
    Sixteen t;
    t.pack(v);
    if (row) t.store(out + (int64_t)m * p.ld + n0);
    if (twice) mirror(p, out, m, n0, lane, t);
    if constexpr (TERMS == 2) {
      float r[16];
      t.rest(v, r);
      t.pack(r);
      if (row) t.store(out + p.term + (int64_t)m * p.ld + n0);
      if (twice) mirror(p, out + p.term, m, n0, lane, t);
    }
  }
}
// Whether a chunk is there to be computed.
template <int KIND>
__device__ __forceinline__ bool wanted(const Params& p, int row0, int n0) {
  return n0 < p.N && (!symmetric(KIND) || (n0 >> 5) <= (row0 >> 5));
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
__global__ void __launch_bounds__(Form<TERMS>::kThreads, 1) muon_umma_kernel(const __grid_constant__ Params p, const __grid_constant__ Maps maps) {
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
      mbar_init(acc_empty + 8 * b, 2 * F::kWarps);
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
  if (!(KIND == kLast && p.step && p.whole == p.tiles)) pdl_launch_dependents();
  pdl_wait();

  Walk walk(pairs, pair);
  Item it;
  auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, p.budget)) != 0; };

  if (TERMS == 2 && warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");  // 4 x 56 + 8 x 224 = 12 x 168, as launched
  if (warp == 0) {
    int s = 0, phase = 0, left_out = blockIdx.x == 0 ? p.drop : -1;
    bool ok = true;
    while (ok && walk.step(p, it)) {
      const Place at = place_of<KIND, F>(p, it.tile);
      const int m0 = at.m * F::kRows + rank * 128, n0 = at.n * F::kCols + rank * 128, halves = halves_of<KIND, F::kWide>(p, at);
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
    const uint32_t idesc = idesc_f16(F::kRows, 256, p.a_mn, p.b_mn);
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
      const int halves = halves_of<KIND, F::kWide>(p, place_of<KIND, F>(p, it.tile));
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
    if constexpr (TERMS == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    constexpr int kPart = 128, kChunks = kPart / 16;  // a warp's columns
    const int quad = warp & 3, part = ((warp - 4) >> 2) & 1, own = (warp - 4) >> 3;  // lanes, columns, accumulator
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const uint32_t empty0 = map_rank(acc_empty, 0), acc = tmem + lanes + own * 256 + kPart * part;
    int full_phase = 0;
    bool ok = true;
    auto wait_full = [&]() {
      const bool there = wait_all(acc_full + 8 * own, full_phase);
      full_phase ^= 1;
      fence_after();
      return there;
    };
    auto give_back = [&](int buffer) {
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty0 + 8 * buffer);
    };
    while (ok && walk.step(p, it)) {
      const Place at = place_of<KIND, F>(p, it.tile);
      if (own >= halves_of<KIND, F::kWide>(p, at)) continue;
      const int row0 = at.m * F::kRows + rank * 128 + 32 * quad;  // this warp's first row
      const bool rows = row0 < p.M;                            // has any: the others only keep step
      const int n_base = at.n * F::kCols + 256 * own + kPart * part;
      float* const piece = it.piece < 0 ? nullptr
                                        : p.partial + (size_t)it.piece * p.piece + (size_t)(rank * 128 + 32 * quad + lane) * F::kCols + 256 * own + kPart * part;
      if (rows && !piece) prefetch<KIND, kPart>(p, at.batch, row0 + lane, n_base);
      const Shared<KIND> all(p, at.batch, row0 + lane);
      if constexpr (TERMS == 2) {
        float sum[16 * kChunks];
#pragma unroll
        for (int i = 0; i < 16 * kChunks; ++i) sum[i] = 0.f;
#pragma unroll 1
        for (int u = it.u0; u < it.u1; u += kRun) {
          ok = wait_full();
          if (!ok) break;
          if (rows) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              float v[16];
              tmem_ld16(acc + 16 * c, v);
              tmem_arrived(v);
#pragma unroll
              for (int i = 0; i < 16; ++i) sum[16 * c + i] += v[i];
            }
          }
          give_back(0);
        }
        if (!ok) break;
        // the last run's commit stands for all products of the tile: the small ones are there too
        if (rows) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            float v[16];
            tmem_ld16(acc + 256 + 16 * c, v);
            tmem_arrived(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[16 * c + i] += v[i];
          }
        }
        give_back(1);
        if (!rows) continue;
        // One copy of the epilogue's code, which takes the first sixteen sums; the others move up.  (Eight copies, each run once a tile, wait
        // for their instructions: 65 us a tile.)
        constexpr bool kEarly = KIND != kForm;  // (four tiles in registers twice are too many)
        Ahead<KIND, TERMS> next;
        if (kEarly && !piece && wanted<KIND>(p, row0, n_base)) next.load(p, at.batch, row0 + lane, n_base);
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
          const int n0 = n_base + 16 * c;
          if (piece) {
            put_piece(piece + 16 * c, sum);
          } else if (wanted<KIND>(p, row0, n0)) {
            if (!kEarly) next.load(p, at.batch, row0 + lane, n0);
            const Ahead<KIND, TERMS> now = next;
            if (kEarly && c + 1 < kChunks && wanted<KIND>(p, row0, n0 + 16)) next.load(p, at.batch, row0 + lane, n0 + 16);
            float more[16];
            beside<KIND, TERMS>(p, all, at.batch, n0, now, more);
            finish<KIND, TERMS>(p, all, at.batch, row0, n0, lane, sum, more);
          }
#pragma unroll
          for (int i = 0; i < 16 * (kChunks - 1); ++i) sum[i] = sum[i + 16];
        }
      } else {
        Ahead<KIND, TERMS> next;
        if (rows && !piece && wanted<KIND>(p, row0, n_base)) next.load(p, at.batch, row0 + lane, n_base);
        ok = wait_full();
        if (!ok) break;
        if (rows && piece) {
#pragma unroll 2
          for (int c = 0; c < kChunks; ++c) {
            float v[16];
            tmem_ld16(acc + 16 * c, v);
            tmem_arrived(v);
            put_piece(piece + 16 * c, v);
          }
        } else if (rows) {
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            const int n0 = n_base + 16 * c;
            if (!wanted<KIND>(p, row0, n0)) break;  // nor is any further one
            const Ahead<KIND, TERMS> now = next;
            float v[16];
            tmem_ld16(acc + 16 * c, v);
            if (c + 1 < kChunks && wanted<KIND>(p, row0, n0 + 16)) next.load(p, at.batch, row0 + lane, n0 + 16);
            float more[16];
            beside<KIND, TERMS>(p, all, at.batch, n0, now, more);
            tmem_arrived(v);
            finish<KIND, TERMS>(p, all, at.batch, row0, n0, lane, v, more);
          }
        }
        give_back(own);
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

// ---- small tiles -----------------------------------------------------------------------------------------------------
// For products that do not fill the device with pairs' tiles: a CTA has one tile of 128 x 64 (or a piece of it along K).  A chain of
// such launches is a chain of latencies (1024 x 256, fp32: 1.8 us from a launch's end to the next one's start, 1.3 to the first K block): up to eight
// pieces are a cluster that joins them through L2; the warps of the epilogue read and multiply what is beside the accumulators while these
// are made, and where the launch leaves SMs idle, all K blocks of a short K are under way at once.  With two terms, every run of K blocks has
// an accumulator of its own, so a piece is at most three runs.
__device__ __forceinline__ void tma_tile_alone(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(c0), "r"(c1),
      "r"(c2), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void umma_alone(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void commit_alone(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

constexpr int small_threads(int warps) { return 64 + 32 * warps; }
// WARPS: of the epilogue: sixteen where a CTA has an SM to itself, eight where two share one.  A whole orthogonalisation with sixteen and with
// eight: fp32 1024 x 256 140 and 147 us, 1024 x 1024 231 and 250, 4096 x 1024 384 and 402; bf16 2048 x 512 132 and 129, 1024 x 1024 150 and 151.
template <int KIND, int TERMS, int WARPS>
__global__ void __launch_bounds__(small_threads(WARPS), 16 / WARPS) muon_small_kernel(const __grid_constant__ Params p, const __grid_constant__ Maps maps) {
  using F = Small<TERMS>;
  constexpr int kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(8) uint64_t bars[2 * kStages + 1];
  volatile int* const abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages;
  if (tid == 0) {
    for (int s = 0; s < 2 * kStages + 1; ++s) mbar_init(full + 8 * s, 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0 && lane < 2 * TERMS) asm volatile("prefetch.tensormap [%0];" ::"l"(lane < TERMS ? &maps.a[lane] : &maps.b[lane - TERMS]) : "memory");
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(F::kTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_slot;
  const bool pieces = p.whole < p.tiles;
  if (!(KIND == kLast && p.step && (!pieces || p.together))) pdl_launch_dependents();
  pdl_wait();

  // pieces of one stretch of K together; a cluster's: of one tile
  const int number = blockIdx.x, part = p.together ? number % p.split : number / p.tiles, tile = p.together ? number / p.split : number - part * p.tiles;
  const Place at = place_of<KIND, F>(p, tile);
  const int u0 = (int)((long long)p.blocks * part / p.split), u1 = (int)((long long)p.blocks * (part + 1) / p.split);
  auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, p.budget)) != 0; };
  if (warp == 0) {
    int s = 0, phase = 0;
    for (int u = u0; u < u1; ++u) {
      if (!wait_all(empty + 8 * s, phase ^ 1)) break;
      if (elect_one()) {
        const int k0 = u * kDeep, m0 = at.m * F::kRows, n0 = at.n * F::kCols;
        const uint32_t bar = full + 8 * s, da = ring + s * F::kStageBytes, db = da + TERMS * kBlockBytes;
        mbar_expect_tx(bar, F::kStageBytes);
        const bool leave = number == 0 && u - u0 == p.drop;
#pragma unroll
        for (int q = 0; q < TERMS; ++q) {
          if (!leave) {
            const uint32_t to = da + q * kBlockBytes;
            if (p.a_mn) {
              tma_tile_alone(to, &maps.a[q], m0, k0, at.batch, bar);
              tma_tile_alone(to + kBlockBytes / 2, &maps.a[q], m0 + 64, k0, at.batch, bar);
            } else {
              tma_tile_alone(to, &maps.a[q], k0, m0, at.batch, bar);
            }
          }
          if (p.b_mn) tma_tile_alone(db + q * F::kBBytes, &maps.b[q], n0, k0, at.batch, bar);
          else tma_tile_alone(db + q * F::kBBytes, &maps.b[q], k0, n0, at.batch, bar);
        }
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; phase ^= 1; }
    }
  } else if (warp == 1) {
    const uint32_t idesc = idesc_f16(F::kRows, F::kCols, p.a_mn, p.b_mn);
    const uint64_t a0 = p.a_mn ? desc_mn_major(ring, kBlockBytes / 2) : desc_k_major(ring);
    const uint32_t ring_b = ring + TERMS * kBlockBytes;
    const uint64_t b0 = p.b_mn ? desc_mn_major(ring_b, F::kBBytes) : desc_k_major(ring_b);
    const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // sixteen k
    int s = 0, phase = 0;
    for (int u = u0; u < u1; ++u) {
      if (!wait_all(full + 8 * s, phase)) break;
      fence_after();
      if (elect_one()) {
        const uint32_t off = (uint32_t)(s * F::kStageBytes) >> 4;
        auto multiply = [&](int buffer, int ta, int tb, uint32_t more) {
#pragma unroll
          for (int k = 0; k < kDeep / 16; ++k)
            umma_alone(tmem + buffer * F::kCols, a0 + off + ta * (kBlockBytes >> 4) + k * a_step, b0 + off + tb * (F::kBBytes >> 4) + k * b_step, idesc,
                       k > 0 ? 1u : more);
        };
        if constexpr (TERMS == 2) {
          multiply(0, 0, 1, u > u0);
          multiply(0, 1, 0, 1);
          multiply(1 + (u - u0) / kRun, 0, 0, (u - u0) % kRun != 0);
        } else {
          multiply(0, 0, 0, u > u0);
        }
        commit_alone(empty + 8 * s);
        if (u + 1 == u1) commit_alone(acc_full);
      }
      __syncwarp();
      if (++s == p.stages) { s = 0; phase ^= 1; }
    }
  } else {
    constexpr int kChunks = 16 / WARPS;  // of sixteen columns, of a warp
    const int quad = warp & 3, across = 16 * kChunks * ((warp - 2) >> 2), n_base = at.n * F::kCols + across, row0 = at.m * F::kRows + 32 * quad;
    const bool rows = row0 < p.M;
    float more[kChunks][16];
    // what this warp finishes: 32 rows and its columns of the tile, or, of a cluster's sixteen parts of 32 x 16, one or none
    const int own = (warp - 2) * p.split + part, own_r = 32 * (own >> 2), own_c = 16 * (own & 3);
    const int joined_row = at.m * F::kRows + own_r, joined_n = at.n * F::kCols + own_c;
    const bool joins = p.together && own < 16 && joined_row < p.M && wanted<KIND>(p, joined_row, joined_n);
    const Shared<KIND> all(p, at.batch, (p.together ? joined_row : row0) + lane);
    if (joins || (rows && !pieces)) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int n0 = p.together ? joined_n : n_base + 16 * c;
        if (c == 1 && (p.together || !wanted<KIND>(p, row0, n0))) break;
        if (c == 0 && !p.together && !wanted<KIND>(p, row0, n0)) break;
        Ahead<KIND, TERMS> a;
        a.load(p, at.batch, (p.together ? joined_row : row0) + lane, n0);
        beside<KIND, TERMS>(p, all, at.batch, n0, a, more[c]);
      }
    }
    if (wait_all(acc_full, 0) && rows) {
      fence_after();
      const uint32_t acc = tmem + ((uint32_t)(32 * quad) << 16) + across;
      float* const piece = p.partial + (size_t)number * p.piece + (size_t)(32 * quad + lane) * F::kCols + across;
#pragma unroll 1
      for (int c = 0; c < kChunks; ++c) {
        const int n0 = n_base + 16 * c;
        if (!pieces && !wanted<KIND>(p, row0, n0)) break;
        float v[16];
        tmem_ld16(acc + 16 * c, v);
        if constexpr (TERMS == 2) {  // the small products first
          float w[16];
          tmem_ld16(acc + F::kCols + 16 * c, w);
          tmem_arrived(v);
          tmem_arrived(w);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] += w[i];
          for (int run = 1; run * kRun < u1 - u0; ++run) {
            tmem_ld16(acc + (1 + run) * F::kCols + 16 * c, w);
            tmem_arrived(w);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += w[i];
          }
        } else {
          tmem_arrived(v);
        }
        if (pieces) {
          put_piece(piece + 16 * c, v);
        } else {
          finish<KIND, TERMS>(p, all, at.batch, row0, n0, lane, v, more[0]);
#pragma unroll
          for (int i = 0; i < 16; ++i) more[0][i] = more[kChunks - 1][i];
        }
      }
    }
    if (p.together) {
      cluster_sync();  // all pieces of the tile are there
      if (joins) {
        float v[16] = {};
        const float* from = p.partial + (size_t)(number - part) * p.piece + (size_t)(own_r + lane) * F::kCols + own_c;
#pragma unroll 4
        for (int q = 0; q < p.split; ++q, from += p.piece) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 f = __ldcg(reinterpret_cast<const float4*>(from) + i);
            v[4 * i] += f.x; v[4 * i + 1] += f.y; v[4 * i + 2] += f.z; v[4 * i + 3] += f.w;
          }
        }
        finish<KIND, TERMS>(p, all, at.batch, joined_row, joined_n, lane, v, more[0]);
      }
    }
  }
  if (p.together && warp < 2) cluster_sync();  // (with the epilogue's warps, above)
  if (*abort_flag)  // (copies and MMAs that may still be in flight end within microseconds)
    for (int i = 0; i < 50; ++i) __nanosleep(1000);
  fence_before();
  __syncthreads();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(F::kTmem) : "memory");
  }
}

// The tiles that were left in pieces: a warp has 32 rows x 16 columns, adds up their pieces in the order of K and does the epilogue.
constexpr int kJoinWarps = 4;
template <int KIND, int TERMS, typename F>
__global__ void __launch_bounds__(32 * kJoinWarps) muon_join_kernel(const __grid_constant__ Params p) {
  const int lane = threadIdx.x & 31, number = blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
  if (!(KIND == kLast && p.step)) pdl_launch_dependents();
  pdl_wait();
  constexpr int kAcross = F::kCols / 16, kPer = kAcross * (F::kRows / 32);
  const int t = number / kPer, in = number % kPer, r0 = in / kAcross * 32, c0 = in % kAcross * 16;
  if (t >= p.tiles - p.whole) return;
  const Place at = place_of<KIND, F>(p, p.whole + t);
  const int row0 = at.m * F::kRows + r0, n0 = at.n * F::kCols + c0;
  if (row0 >= p.M || !wanted<KIND>(p, row0, n0)) return;
  Ahead<KIND, TERMS> now;
  now.load(p, at.batch, row0 + lane, n0);
  const Shared<KIND> all(p, at.batch, row0 + lane);
  float v[16] = {}, more[16];
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
  beside<KIND, TERMS>(p, all, at.batch, n0, now, more);
  finish<KIND, TERMS>(p, all, at.batch, row0, n0, lane, v, more);
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
int tiles_of(int kind, int rows, int cols, int M, int N, int* m_tiles = nullptr, int* n_tiles = nullptr) {
  const int m = (M + rows - 1) / rows, n = (N + cols - 1) / cols;
  if (m_tiles) *m_tiles = m;
  if (n_tiles) *n_tiles = n;
  if (!symmetric(kind)) return m * n;
  if (cols <= rows) return rows / cols * (m * (m - 1) / 2) + n;
  return m / 2 * (m / 2 + 1) + (m & 1 ? m / 2 + 1 : 0);
}

constexpr double kTogether = 4.5;  // microseconds of a cluster that joins its pieces
struct Plan {
  int per, m_tiles, n_tiles, tiles, whole, split, ctas, stages, together;
  double time;
};
// Floats of the pieces that the workspace has room for: 84 MB.
constexpr size_t kPieceFloats = (size_t)160 * 256 * 512;
long long most_pieces(int rows, int cols, long long tiles, long long blocks) {
  const long long room = (long long)(kPieceFloats / ((size_t)rows * cols));
  return tiles < room && tiles * blocks < room ? tiles * blocks : room;
}
// Microseconds of the launch that joins `split` pieces of each of so many tiles.
double join_time(double tiles, int split, int rows, int cols) { return 4.0 + 0.2 * split + tiles * (split + 1) * rows * cols * 4 / 2e6; }

// Pairs' tiles: whole ones in rounds, the last, partly idle one cut along K into equal pieces where that is shorter (times in microseconds: of
// a K block, of a tile's epilogue, of a piece's way to the workspace).
template <int TERMS>
Plan plan_pairs(int kind, int M, int N, int K, int n, int pairs) {
  using F = Form<TERMS>;
  Plan p{};
  p.per = tiles_of(kind, F::kRows, F::kCols, M, N, &p.m_tiles, &p.n_tiles);
  p.tiles = p.per * n;
  const int blocks = (K + kDeep - 1) / kDeep, rest = p.tiles % pairs;
  const double block = TERMS == 1 ? 0.7 : 1.2, start = 3.0, tail = TERMS == 1 ? 15.0 : 24.0, piece = TERMS == 1 ? 3.0 : 2.0;
  const long long room = most_pieces(F::kRows, F::kCols, p.tiles, blocks);
  // two terms: a tile's epilogue runs under the next one's products
  const double rounds = start + (double)(p.tiles / pairs) * (TERMS == 2 ? std::max(blocks * block, tail) : blocks * block + tail);
  p.whole = p.tiles;
  p.split = 1;
  p.time = rounds + (rest > 0 ? blocks * block + tail : TERMS == 2 ? tail : 0.0);
  for (int split = 1; rest > 0 && split <= blocks && (long long)rest * split <= room; ++split) {
    const int turns = (rest * split + pairs - 1) / pairs;
    const double time = rounds + turns * (std::ceil((double)blocks / split) * block + piece) + join_time(rest, split, F::kRows, F::kCols);
    if (time < p.time) {
      p.time = time;
      p.whole = p.tiles - rest;
      p.split = split;
    }
  }
  const int pieces = (p.tiles - p.whole) * p.split, most = p.whole > pieces ? p.whole : pieces;
  p.ctas = 2 * (most < pairs ? most : pairs);
  return p;
}
// Small tiles: whole, or all of them in pieces.
template <int TERMS>
Plan plan_small(int kind, int M, int N, int K, int n, int sms) {
  using F = Small<TERMS>;
  Plan p{};
  p.per = tiles_of(kind, F::kRows, F::kCols, M, N, &p.m_tiles, &p.n_tiles);
  p.tiles = p.per * n;
  const int blocks = (K + kDeep - 1) / kDeep, fewest = (blocks + F::kMostBlocks - 1) / F::kMostBlocks;
  const long long room = most_pieces(F::kRows, F::kCols, p.tiles, blocks);
  p.time = 1e30;
  // A CTA with all stages fills an SM, half as many leave room for another.  Two, four or eight pieces are a cluster, which joins them itself: an
  // SM each, clusters find about 128 places (those of eight two in a part of the device of 16 to 20 SMs).
  const int alone = sms, clustered = sms * 7 / 8;
  for (int split = fewest; split <= blocks && (split == 1 || (long long)p.tiles * split <= room); ++split) {
    const bool together = split > 1 && split <= 8;
    if (together && (split & (split - 1))) continue;
    const long long ctas = (long long)p.tiles * split;
    if (ctas > (1 << 30)) break;
    const int places = together ? clustered : alone;
    const bool full = ctas <= places;
    const long long rounds = full ? 1 : (ctas + 2 * places - 1) / (2 * places);
    const double block = (TERMS == 1 ? 0.3 : 0.65) * (full ? 1 : 2);  // two CTAs share an SM's copies
    const double joined = split == 1 ? 0.0 : together ? kTogether : join_time(p.tiles, split, F::kRows, F::kCols);
    const double time = 3.0 + rounds * (2.0 + std::ceil((double)blocks / split) * block + (split > 1 ? 1.0 : 3.0)) + joined;
    if (time < p.time) {
      p.time = time;
      p.split = split;
      p.together = together;
      p.stages = full ? F::kStages : F::kStages / 2;
    }
  }
  p.whole = p.split > 1 ? 0 : p.tiles;
  p.ctas = p.tiles * p.split;
  return p;
}

template <int KIND, int TERMS, typename F>
cudaError_t launch_join(const Params& p, cudaStream_t s) {
  const int warps = (p.tiles - p.whole) * (F::kCols / 16) * (F::kRows / 32);
  return launch_pdl(muon_join_kernel<KIND, TERMS, F>, dim3((warps + kJoinWarps - 1) / kJoinWarps), dim3(32 * kJoinWarps), 0, s, p);
}
template <typename F>
void take_plan(Params& p, const Plan& plan) {
  p.m_tiles = plan.m_tiles; p.n_tiles = plan.n_tiles; p.per = plan.per; p.tiles = plan.tiles; p.whole = plan.whole; p.split = plan.split;
  p.stages = plan.stages;
  p.together = plan.together;
  p.blocks = (p.K + kDeep - 1) / kDeep;
  p.piece = F::kRows * F::kCols;
}
template <int KIND, int TERMS>
cudaError_t launch_pairs(Params& p, const Plan& plan, const Maps& maps, cudaStream_t s) {
  using F = Form<TERMS>;
  take_plan<F>(p, plan);
  static unsigned long long configured = 0;
  cudaError_t e = allow_dynamic_smem(muon_umma_kernel<KIND, TERMS>, F::kSmemBytes, configured);
  if (e != cudaSuccess) return e;
  if constexpr (TERMS == 2) {  // the registers that the roles share out have to be there: a warp that asks for more than there are waits for ever
    static const bool enough = [] {
      cudaFuncAttributes a;
      return cudaFuncGetAttributes(&a, muon_umma_kernel<KIND, TERMS>) == cudaSuccess && a.numRegs >= 168;
    }();
    if (!enough) return cudaErrorInvalidConfiguration;
  }
  e = launch_clusters(2, muon_umma_kernel<KIND, TERMS>, dim3(plan.ctas), dim3(F::kThreads), F::kSmemBytes, s, p, maps);
  return e != cudaSuccess || p.whole == p.tiles ? e : launch_join<KIND, TERMS, F>(p, s);
}
template <int KIND, int TERMS, int WARPS>
cudaError_t launch_small(Params& p, const Plan& plan, const Maps& maps, cudaStream_t s) {
  using F = Small<TERMS>;
  take_plan<F>(p, plan);
  static unsigned long long configured = 0;
  cudaError_t e = allow_dynamic_smem(muon_small_kernel<KIND, TERMS, WARPS>, F::smem_bytes(F::kStages), configured);
  if (e != cudaSuccess) return e;
  e = launch_clusters(plan.together ? plan.split : 1, muon_small_kernel<KIND, TERMS, WARPS>, dim3(plan.ctas), dim3(small_threads(WARPS)), F::smem_bytes(plan.stages), s, p, maps);
  return e != cudaSuccess || p.whole == p.tiles || p.together ? e : launch_join<KIND, TERMS, F>(p, s);
}

// What a product's operands are, and how they lie: `k`: rows are k.
struct Operand {
  const uint16_t* data;
  int64_t width, rows, ld, matrix, term;
  bool k;
};

template <int KIND, int TERMS>
cudaError_t launch(const MuonBatch& b, Params& p, const Operand& x, const Operand& y, int sm_count, cudaStream_t s) {
  const Plan pairs = plan_pairs<TERMS>(KIND, p.M, p.N, p.K, b.n, sm_count / 2 < kMuonPairs ? sm_count / 2 : kMuonPairs);
  const Plan alone = plan_small<TERMS>(KIND, p.M, p.N, p.K, b.n, sm_count);
  const bool few = alone.time < pairs.time;
  Maps maps;
  for (int t = 0; t < TERMS; ++t) {
    auto make = [&](CUtensorMap* m, const Operand& o, int rows) { return make_map(m, o.data + t * o.term, o.width, o.rows, o.ld, b.n, o.matrix, o.k ? 64 : rows); };
    if (!make(&maps.a[t], x, 128) || !make(&maps.b[t], y, few ? 64 : 128)) return cudaErrorInvalidValue;
  }
  if (TERMS == 1) maps.a[1] = maps.a[0], maps.b[1] = maps.b[0];
  p.a_mn = x.k;
  p.b_mn = y.k;
  if (!few) return launch_pairs<KIND, TERMS>(p, pairs, maps, s);
  return alone.stages == Small<TERMS>::kStages ? launch_small<KIND, TERMS, 16>(p, alone, maps, s) : launch_small<KIND, TERMS, 8>(p, alone, maps, s);
}

}  // namespace

size_t muon_partial_floats(int S, int R, int C, int n, int terms) {
  size_t most = 0;
  const int sizes[2][2] = {{Form<1>::kRows, terms == 1 ? Form<1>::kCols : Form<2>::kCols}, {Small<1>::kRows, Small<1>::kCols}};
  for (const auto& size : sizes) {
    for (int kind : {kGram, kForm, kApply}) {
      const long long K = kind == kGram ? (R > C ? R : C) : S, blocks = (K + kDeep - 1) / kDeep;
      const long long tiles = (long long)tiles_of(kind, size[0], size[1], kind == kApply ? R : S, kind == kApply ? C : S) * n;
      const size_t floats = (size_t)most_pieces(size[0], size[1], tiles, blocks) * size[0] * size[1];
      if (floats > most) most = floats;
    }
  }
  return most;
}

cudaError_t launch_muon_product(const MuonBatch& b, const MuonProduct& q, int sm_count, cudaStream_t s) {
  Params p{};
  p.S = b.S;
  const bool sym = symmetric(q.kind);
  p.M = sym ? b.S : b.R;
  p.N = sym ? b.S : b.C;
  p.K = q.kind == kGram ? b.L : b.S;
  p.partial = b.partial;
  p.status = b.status;
  p.budget = fused_test_knobs().wait_cycles;
  p.drop = fused_test_knobs().drop_stage;
  p.tall = b.tall;
  p.first = q.first;
  p.factors = b.first;
  p.ld = sym ? b.ld_p : b.ld_x;
  p.matrix = sym ? b.p_matrix : b.x_matrix;
  p.term = sym ? b.p_term : b.x_term;
  auto two = [](int e) { return (float)std::ldexp(1.0, e); };
  auto diag = [&](int i) { return b.diag + (size_t)i * b.n * ((b.S + 15) / 16 * 16); };
  const uint16_t* const X = b.x[q.from];
  auto square = [&](int i) { return Operand{b.sym[i], b.S, b.S, b.ld_p, b.p_matrix, b.p_term, false}; };
  auto long_side = [&](bool k) { return Operand{X, b.C, b.R, b.ld_x, b.x_matrix, b.x_term, k}; };
  if (q.kind == kGram) {
    p.k = two(q.e_out - 2 * q.ex);
    p.dacc = two(-2 * q.ex);
    p.out = b.sym[q.out];
    p.out_diag = diag(q.out);
    const Operand x = long_side(b.tall);  // rows of X are k where it is tall
    return b.terms == 1 ? launch<kGram, 1>(b, p, x, x, sm_count, s) : launch<kGram, 2>(b, p, x, x, sm_count, s);
  }
  if (q.kind == kForm) {
    const bool same = q.m.which == q.n.which;
    p.out = b.sym[q.out];
    p.out_diag = diag(q.out);
    p.M_ = b.sym[q.m.which];
    p.M_diag = diag(q.m.which);
    p.N_ = same ? nullptr : b.sym[q.n.which];
    p.N_diag = diag(q.n.which);
    p.m = q.m.c * two(q.e_out - q.m.e);
    p.nn = q.n.c * two(q.e_out - q.n.e);
    p.k_m = q.k.c * two(q.e_out - q.m.e);
    p.k_n = q.k.c * two(q.e_out - q.n.e);
    p.k = q.k.c * two(q.e_out - q.m.e - q.n.e);
    p.dm = q.m.c; p.dn = q.n.c; p.dk = q.k.c;
    p.dacc = two(-q.m.e - q.n.e);
    p.fm = q.m.factor; p.fn = q.n.factor; p.fk = q.k.factor;
    const Operand m = square(q.m.which), n = square(q.n.which);
    return b.terms == 1 ? launch<kForm, 1>(b, p, m, n, sm_count, s) : launch<kForm, 2>(b, p, m, n, sm_count, s);
  }
  const bool last = q.kind == kLast;
  const Operand x = b.tall ? long_side(false) : square(q.m.which), y = b.tall ? square(q.m.which) : long_side(true);
  p.q = q.k.c;
  p.fq = q.k.factor;
  p.x_scale = two((last ? 0 : q.e_out) - q.ex);
  p.acc_scale = two((last ? 0 : q.e_out) - q.ex - q.m.e);
  p.diag = diag(q.m.which);
  p.both = b.terms == 2 || q.late;
  p.X = X;
  if (!last) {
    p.out = b.x[q.from ^ 1];
    return b.terms == 1 ? launch<kApply, 1>(b, p, x, y, sm_count, s) : launch<kApply, 2>(b, p, x, y, sm_count, s);
  }
  p.step = b.step;
  p.out_bf16 = b.out_bf16;
  p.grad_norm = b.grad_norm;
  for (int i = 0; i < b.n; ++i) p.item[i] = b.item[i];
  return b.terms == 1 ? launch<kLast, 1>(b, p, x, y, sm_count, s) : launch<kLast, 2>(b, p, x, y, sm_count, s);
}

}  // namespace sffn
