// Training form of the gated FFN: what the host side (train_api.cu) hands to the kernels, and the element-wise part that
// every product's epilogue shares.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "sparse_ffn.h"

namespace sffn {

// A product C[m, n] = sum_k A(m, k) B(n, k), and what becomes of C.
//   kStore   out = C
//   kGateUp  two products over one A: z = C_0 + bias, u = C_1; stores z, u (if wanted) and h = A(z) . A_3(u)
//   kHidden  C = dh: reads z, u; stores dz, du, h and sums dz over its rows into one line of `db`
enum { kEpiStore = 0, kEpiGateUp = 1, kEpiHidden = 2 };

// An operand as it lies in memory: `major_k`: rows are m (or n), consecutive elements k; else rows are k, consecutive
// elements m (or n).  `ld`: elements between rows.
struct TrainOperand {
  const void* data;
  int64_t ld;
};

struct TrainEpilogue {
  int M, N;                // of C
  int act, act_up;
  const float* bias;       // [N] or NULL
  void* out[3];            // kStore: of product 0, 1, 2 of a batch
  int64_t ld_out;
  void *z, *u;             // the caller's [M, N]
  int64_t ld_zu;
  void *h, *dz, *du;       // workspace [M, ld_h], NULL where not wanted
  int64_t ld_h;
  int64_t limb;            // tensor-core kernels, fp32 storage: h, dz, du are three bf16 matrices, so many elements apart
  float* db;               // [lines, ld_h] partial sums of dz, NULL where not wanted
};

struct TrainGemm {
  int M, N, K;
  int parts;               // kStore: products that are added up (1 or 2); kGateUp: 2 with one A
  int batch;               // kStore: independent products of one shape (1 to 3)
  TrainOperand a[3], b[3];
  bool a_major_k, b_major_k;
  int epilogue;
  TrainEpilogue epi;
};

// An activation's value and slope.  FAST: the hardware's exponential and division (errors of 1e-6, under bf16 storage).
template <bool FAST>
__device__ __forceinline__ float train_sigmoid(float t) {
  return FAST ? __fdividef(1.f, 1.f + __expf(-t)) : 1.f / (1.f + expf(-t));
}
template <bool FAST>
__device__ __forceinline__ float train_act(int act, float t) {
  if (act == kActNone) return t;
  const float p = fmaxf(t, 0.f);
  if (act == kActRelu) return p;
  if (act == kActSqRelu) return p * p;
  const float r = act == kActSilu ? t : p;
  return r * train_sigmoid<FAST>(r);
}
template <bool FAST>
__device__ __forceinline__ void train_act_slope(int act, float t, float& value, float& slope) {
  if (act == kActNone) { value = t; slope = 1.f; return; }
  const bool on = t > 0.f;
  if (act == kActRelu) { value = on ? t : 0.f; slope = on ? 1.f : 0.f; return; }
  if (act == kActSqRelu) { const float p = on ? t : 0.f; value = p * p; slope = 2.f * p; return; }
  const float s = train_sigmoid<FAST>(t);
  const bool keep = act == kActSilu || on;
  value = keep ? t * s : 0.f;
  slope = keep ? fmaf(t * s, 1.f - s, s) : 0.f;
}

// Small products in fp32 FMAs (train_simt.cu), fp32 operands.  *lines: of partial sums that kHidden leaves in `db`, at most
// train_simt_lines(M).
int train_simt_lines(int M);
cudaError_t launch_train_simt(const TrainGemm& g, int* lines, cudaStream_t s);
// Plain products of small K whose operands both lie with K as rows (train_outer.cu), rows of A padded to a multiple of eight
// values, operands as they are stored (no terms), K at most kOuterF32 / kOuterBf16.
constexpr int kOuterF32 = 16, kOuterBf16 = 4;
cudaError_t launch_train_outer(const TrainGemm& g, int dtype, cudaStream_t s);
// db_g[j] = sum over `lines` lines of partial sums, in order; 0 for no line.
cudaError_t launch_train_column_sums(const float* partial, int lines, int64_t ld, int N, float* out, cudaStream_t s);

// Tensor-core kernels (train_umma.cu).  Operands are bf16 matrices or, for fp32 storage, three bf16 matrices each (`limb`
// elements apart) that add up to it; all on 16 bytes, rows a multiple of 16 bytes apart.
struct TrainUmma {
  TrainGemm g;
  bool f32;                // storage type of the outputs, and three terms an operand
  int64_t limb_a[3], limb_b[3];
  float* partial;          // room for the pieces of tiles that several pairs of CTAs share (train_umma_partial_bytes)
  int32_t* status;
};
constexpr int kTrainUmmaPairs = 80;    // pairs of CTAs at most
constexpr int kTrainPieces = 2 * kTrainUmmaPairs;  // of tiles that are cut, at most
// The most that the pieces of a product M x N may take, on any device: `blocks` of K, in 64s, of all parts.
size_t train_umma_partial_bytes(int epilogue, bool f32, int M, int N, long long blocks, int batch);
int train_umma_lines(int M);
cudaError_t launch_train_umma(const TrainUmma& t, cudaStream_t s);
// out[l][r][c], l = 0, 1, 2: the bf16 terms of in[r][c]; `ld_out` elements between rows, `limb` between terms.
cudaError_t launch_train_split(const float* in, int64_t ld_in, int rows, int cols, __nv_bfloat16* out, int64_t ld_out, int64_t limb, cudaStream_t s);

}  // namespace sffn
