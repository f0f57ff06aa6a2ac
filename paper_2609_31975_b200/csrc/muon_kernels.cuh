// The orthogonalised update and the Muon step: what the host side (muon_api.cu) hands to the kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "sparse_ffn.h"

namespace sffn {

constexpr int kMuonBatch = 64;     // matrices of a launch, at most
constexpr int kMuonPartials = 1024; // partial sums of a matrix's squares, at most
constexpr int kMuonPairs = 80;     // pairs of CTAs at most

// A matrix as the caller has it.
struct MuonItem {
  const void* src;      // the update, or the gradient
  int64_t ld_src;
  void* out;            // the orthogonal matrix, or the parameter
  int64_t ld_out;
  float *m, *master;    // step: moments, copy in 32 bits or NULL
  float decay, rate;    // step: p = decay p - rate O
};

// A batch of matrices of one shape and the workspace that they share.  Matrices are fp16, a value v standing as v 2^e: X [R, C] in two
// terms (hi and what it leaves), A = X X^T (or X^T X) and polynomials of it [S, S] in `terms`, without their diagonals, which are fp32.
struct MuonBatch {
  MuonItem item[kMuonBatch];
  int n;                // matrices
  int R, C, S, L;       // rows, columns, shorter and longer side
  bool tall;            // R > C: P = X^T X
  bool step, nesterov, src_bf16, out_bf16;
  int terms;            // of the products' operands
  float momentum, one_momentum, eps;
  const float* grad_norm;
  float max_norm;
  // workspace
  int64_t ld_x, ld_p;   // elements
  int64_t x_matrix, p_matrix, x_term, p_term;  // elements between matrices of a batch, and between terms
  uint16_t *x[2], *sym[4];
  float* diag;          // [4][n, S up to a multiple of 16]: the diagonals of sym
  float* first;         // [n][4]: g, g^2, g^3, g^5: the first X is g times what is stored
  double* squares;      // [n][kMuonPartials]
  float* partial;       // pieces of tiles that are cut
  int32_t* status;
};

// A product and its epilogue.
//   kGram   A = X X^T (X^T X) into sym[out]
//   kForm   sym[out] = m M + n N + k M N, polynomials of A; out is neither M nor N
//   kApply  X' = k X + M X (X M); X is x[from], X' the other one
//   kLast   the same into the caller's matrix
enum { kGram = 0, kForm = 1, kApply = 2, kLast = 3 };
__host__ __device__ constexpr bool symmetric(int kind) { return kind == kGram || kind == kForm; }
struct MuonTerm {
  int which;            // of sym
  int e;                // the exponent that it is stored with
  float c;              // coefficient,
  int factor;           // and which of the first step's factors multiplies it (-1: none)
};
struct MuonProduct {
  int kind, from, out;
  bool first;           // factors are to be looked at
  MuonTerm m, n, k;
  int ex, e_out;        // exponents that X, and the result, are stored with
  bool late;            // the steps to come multiply small singular values by four at most
};

cudaError_t launch_muon_product(const MuonBatch& b, const MuonProduct& p, int sm_count, cudaStream_t s);
// Floats that the pieces of a batch's products may take, on any device.
size_t muon_partial_floats(int S, int R, int C, int n, int terms);

// Moments (step), and the squares' sums; then X = U 2^k in two terms, with its factor.
cudaError_t launch_muon_moments(const MuonBatch& b, int sm_count, cudaStream_t s);
cudaError_t launch_muon_scale(const MuonBatch& b, int sm_count, cudaStream_t s);
constexpr int kMuonExponent = 14;  // X before the first step: norm 2^13 to 2^14 as stored

}  // namespace sffn
