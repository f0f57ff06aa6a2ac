// Shared by the tensor-core kernels of the training calls (train_umma.cu, train_umma_f32.cu): what a launch is given, how its
// tiles are dealt to pairs of CTAs, and element-wise parts of the epilogues.
#pragma once

#include "tcgen05.cuh"
#include "train_kernels.cuh"

namespace sffn {

constexpr int kPairRows = 256;               // rows of a pair's tile
constexpr int kDeep = 64;                    // bf16 elements of one 128-byte swizzle row: a K block
constexpr int kHalfBytes = 128 * kDeep * 2;  // 128 rows of a K block
constexpr int kLimbProducts = 6;             // fp32: products of a K block
constexpr int kLimbRun = 2;                  // K blocks of a run
constexpr int kRunBlocks = 12;               // dh: K blocks of a run


struct UmmaParams {
  TrainEpilogue epi;
  int m_tiles, n_tiles, tiles;        // tiles = m_tiles * n_tiles * batch
  int blocks;                         // K blocks of a part
  int units, run_units;               // a tile's K blocks, those of a run
  int whole;                          // tiles dealt whole; the others are cut along K,
  int split;                          // into so many pieces each
  int batch, tile_cols;
  int a_mn, b_mn;
  int a_rows, stages, stage_bytes;    // bf16: rows of A that a CTA copies; the ring
  float* partial;
  size_t piece;                       // floats of a piece
  int32_t* status;
  long long budget;
  int drop;                           // test hook: a K block whose rows of A CTA 0 leaves out, so that the wait for them runs out (-1: none)
};

// One piece of work of a pair of CTAs: units [u0, u1) of a tile, whose sums go to the workspace as piece number `piece` (-1: a whole tile).
struct Item {
  int tile, u0, u1, piece;
};
// A pair's items in order: pieces of the tiles that are cut (the first pieces of all, then the second ones ..: what runs at one time
// is of one stretch of K, whose rows and columns the tiles share in L2), then whole tiles.
struct Walk {
  int pairs, next_piece, next;
  __device__ __forceinline__ Walk(const UmmaParams& p, int pairs_, int pair) : pairs(pairs_), next_piece(pair), next(pair) {}
  __device__ __forceinline__ bool step(const UmmaParams& p, Item& it) {
    const int cut = p.tiles - p.whole;
    if (next_piece < cut * p.split) {
      const int part = next_piece / cut;
      it.tile = p.whole + next_piece - part * cut;
      it.u0 = p.units * part / p.split;
      it.u1 = p.units * (part + 1) / p.split;
      it.piece = next_piece;
      next_piece += pairs;
      return true;
    }
    if (next >= p.whole) return false;
    it.tile = next;
    it.u0 = 0;
    it.u1 = p.units;
    it.piece = -1;
    next += pairs;
    return true;
  }
};

// Where a tile lies: groups of eight tile rows, column by column, so that what runs at one time shares rows and columns in L2.
struct Place {
  int batch, m, n;
};
__device__ __forceinline__ Place place_of(const UmmaParams& p, int tile) {
  constexpr int kGroup = 8;
  const int per = p.m_tiles * p.n_tiles;
  Place at;
  at.batch = tile / per;
  tile -= at.batch * per;
  const int group = tile / (kGroup * p.n_tiles), first = group * kGroup, rows = min(kGroup, p.m_tiles - first);
  tile -= first * p.n_tiles;
  at.m = first + tile % rows;
  at.n = tile / rows;
  return at;
}

// Rows and columns of a tile's accumulators that a piece holds: the rows that there are, in 32s (what the epilogue's warps look at).
__host__ __device__ constexpr int piece_rows(int M) { return M < kPairRows ? (M + 31) / 32 * 32 : kPairRows; }
__host__ __device__ constexpr int piece_cols(int epilogue, bool f32) { return epilogue == kEpiStore && !f32 ? 512 : 256; }
// A piece, [rows][columns of the accumulators] fp32: part `part` of the t-th tile that is cut is number t + part * (tiles that are cut).
__device__ __forceinline__ float* piece_of(const UmmaParams& p, int number) { return p.partial + (size_t)number * p.piece; }
// Sixteen columns of a row of a piece.
__device__ __forceinline__ void put_piece(float* at, const float* v) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(at + 8 * h), "f"(v[8 * h]), "f"(v[8 * h + 1]), "f"(v[8 * h + 2]), "f"(v[8 * h + 3]),
                 "f"(v[8 * h + 4]), "f"(v[8 * h + 5]), "f"(v[8 * h + 6]), "f"(v[8 * h + 7])
                 : "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Activations of sixteen values, the choice made once: inside the loops it would be made, and its code be there, sixteen times.
template <bool FAST>
__device__ __forceinline__ void act16(int act, const float* t, float* v) {
  if (act == kActNone) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = t[i];
  } else if (act == kActRelu) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActRelu, t[i]);
  } else if (act == kActSqRelu) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActSqRelu, t[i]);
  } else if (act == kActRsPlus) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActRsPlus, t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActSilu, t[i]);
  }
}
template <bool FAST, int ACT, typename Raw>
__device__ __forceinline__ void slope16_of(const Raw& t, float* v, float* d) {
#pragma unroll
  for (int i = 0; i < 16; ++i) train_act_slope<FAST>(ACT, t.get(i), v[i], d[i]);
}
template <bool FAST, typename Raw>
__device__ __forceinline__ void slope16(int act, const Raw& t, float* v, float* d) {
  if (act == kActNone) slope16_of<FAST, kActNone>(t, v, d);
  else if (act == kActRelu) slope16_of<FAST, kActRelu>(t, v, d);
  else if (act == kActSqRelu) slope16_of<FAST, kActSqRelu>(t, v, d);
  else if (act == kActRsPlus) slope16_of<FAST, kActRsPlus>(t, v, d);
  else slope16_of<FAST, kActSilu>(t, v, d);
}

// Sums of sixteen columns over the lanes of a warp: lanes 2 i and 2 i + 1 get column i's (in halves of what is left, five
// exchanges deep, sixteen shuffles).
__device__ __forceinline__ float column_sum(float* v, int lane) {
#pragma unroll
  for (int width = 8; width >= 1; width >>= 1) {
    const bool upper = lane & (2 * width);
#pragma unroll
    for (int i = 0; i < width; ++i) {
      const float send = upper ? v[i] : v[i + width], keep = upper ? v[i + width] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, 2 * width);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

// ---- host ------------------------------------------------------------------------------------------------------------

// `terms` bf16 matrices [rows, width], rows `ld` elements apart, in boxes of 64 elements x `box` rows, 128-byte swizzle.
bool make_train_map(CUtensorMap* m, const void* base, int64_t width, int64_t rows, int64_t ld, int terms, int64_t limb, int box);
// The maps of a product's operands, three of each (the first one again where there are fewer); a_rows: of a box of a K-major A.
bool make_operand_maps(const TrainUmma& t, int a_rows, CUtensorMap* a, CUtensorMap* b);
// Fills in what follows from the product: tiles of `cols` columns, K in units, which tiles are cut for `pairs` pairs of CTAs
// (returned: the pairs that have work).
int plan_umma(const TrainUmma& t, int cols, UmmaParams& p, int pairs);

cudaError_t launch_train_umma_f32(const TrainUmma& t, int pairs, cudaStream_t s);
// The epilogue of the tiles that were cut along K, after the launch that left their pieces.
cudaError_t launch_train_join(const UmmaParams& p, int epilogue, bool f32, cudaStream_t s);

}  // namespace sffn
