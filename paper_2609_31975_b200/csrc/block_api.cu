// Host side of the norms around a block: argument checks.
#include <cmath>

#define SFFN_FILE "block_api.cu"
#include "block_kernels.cuh"
#include "host_checks.cuh"
#include "sparse_ffn.h"

using namespace sffn::host;

namespace {

constexpr int kMaxTokens = 1 << 30;  // a grid's rows

int check_shape(int D, int y_dtype, int h_dtype, int n_dtype) {
  if (D <= 0 || !storage_type(y_dtype) || !storage_type(h_dtype) || !storage_type(n_dtype)) return SFFN_ERR_INVALID_ARG;
  const bool half = y_dtype == SFFN_BF16 || h_dtype == SFFN_BF16 || n_dtype == SFFN_BF16;
  return D > SFFN_BLOCK_MAX_D || D % (half ? 8 : 4) ? SFFN_ERR_UNSUPPORTED : SFFN_OK;
}

// What both passes read.
int check_call(const sffn_block_norm* c) {
  if (!c || c->T < 0) return SFFN_ERR_INVALID_ARG;
  const int shape = check_shape(c->D, c->y_dtype, c->h_dtype, c->n_dtype);
  if (shape != SFFN_OK) return shape;
  if (c->T > kMaxTokens) return SFFN_ERR_UNSUPPORTED;
  if (c->gate_kind < SFFN_BLOCK_GATE_NONE || c->gate_kind > SFFN_BLOCK_GATE_FULL || !std::isfinite(c->scale) || !(c->eps >= 0) || std::isinf(c->eps)) return SFFN_ERR_INVALID_ARG;
  if (c->T > 0 && !c->y && (c->gate_kind != SFFN_BLOCK_GATE_NONE || c->post_gain)) return SFFN_ERR_INVALID_ARG;
  if (!aligned(c->post_gain, 16) || !aligned(c->pre_gain, 16) || !aligned(c->stats, 4)) return SFFN_ERR_UNSUPPORTED;
  if (c->gate_kind == SFFN_BLOCK_GATE_NONE) return SFFN_OK;
  if (!c->gate && (c->T > 0 || c->gate_kind == SFFN_BLOCK_GATE_CHANNEL)) return SFFN_ERR_INVALID_ARG;
  if (c->gate_kind == SFFN_BLOCK_GATE_FULL) return c->T > 0 ? check_rows(c->gate, c->ld_gate, c->D, element(c->h_dtype)) : SFFN_OK;
  return aligned(c->gate, c->gate_kind == SFFN_BLOCK_GATE_CHANNEL ? 16 : 4) ? SFFN_OK : SFFN_ERR_UNSUPPORTED;
}

Span rows_of(const void* p, int64_t T, int64_t D, int dtype, int64_t ld) {
  const int64_t e = (int64_t)element(dtype);
  return {p, T, e * D, e * ld};
}
Span gate_of(const sffn_block_norm* c, const void* p, int64_t ld) {
  return c->gate_kind == SFFN_BLOCK_GATE_NONE ? Span{nullptr, 0, 0, 0}
         : c->gate_kind == SFFN_BLOCK_GATE_FULL ? rows_of(p, c->T, c->D, c->h_dtype, ld) : whole(p, 4ll * (c->gate_kind == SFFN_BLOCK_GATE_CHANNEL ? c->D : c->T));
}
// An output that may lie over an input exactly is left out of the comparison with it.
bool same(const Span& a, const Span& b) { return a.p == b.p && (a.ld == b.ld || a.rows <= 1); }

}  // namespace

extern "C" {

int sffn_block_norm_forward(const sffn_block_norm* c, void* stream) {
  const int rc = check_call(c);
  if (rc != SFFN_OK) return rc;
  if (c->T == 0) return SFFN_OK;  // (tensors without rows have no address)
  if ((!c->y && (!c->resid || !c->pre_gain)) || (c->y && !c->h) || (c->pre_gain && !c->n)) return SFFN_ERR_INVALID_ARG;
  const size_t ey = element(c->y_dtype), eh = element(c->h_dtype), en = element(c->n_dtype);
  int rows = c->y ? check_rows(c->y, c->ld_y, c->D, ey) : SFFN_OK;
  if (rows == SFFN_OK && c->resid) rows = check_rows(c->resid, c->ld_resid, c->D, eh);
  if (rows == SFFN_OK && c->y) rows = check_rows(c->h, c->ld_h, c->D, eh);
  if (rows == SFFN_OK && c->pre_gain) rows = check_rows(c->n, c->ld_n, c->D, en);
  if (rows != SFFN_OK) return rows;
  const Span y = rows_of(c->y, c->T, c->D, c->y_dtype, c->ld_y), resid = rows_of(c->resid, c->T, c->D, c->h_dtype, c->ld_resid);
  const Span h = c->y ? rows_of(c->h, c->T, c->D, c->h_dtype, c->ld_h) : Span{nullptr, 0, 0, 0};
  const Span n = c->pre_gain ? rows_of(c->n, c->T, c->D, c->n_dtype, c->ld_n) : Span{nullptr, 0, 0, 0}, stats = whole(c->stats, 8ll * c->T);
  if (outputs_meet({y, gate_of(c, c->gate, c->ld_gate), whole(c->post_gain, 4ll * c->D), whole(c->pre_gain, 4ll * c->D)}, {h, n, stats}) || meet(n, resid) ||
      meet(stats, resid) || (meet(h, resid) && !same(h, resid)))
    return SFFN_ERR_INVALID_ARG;
  int sms = 0;
  const int count = sm_count(&sms);
  if (count != SFFN_OK) return count;
  SFFN_CUDA(sffn::launch_block_forward(*c, sms, static_cast<cudaStream_t>(stream)));
  return SFFN_OK;
}

int sffn_block_norm_workspace_bytes(int D, size_t* bytes) {
  if (!bytes) return SFFN_ERR_INVALID_ARG;
  const int shape = check_shape(D, SFFN_F32, SFFN_F32, SFFN_F32);
  if (shape != SFFN_OK) return shape;
  *bytes = (size_t)2 * sffn::block_lines(D) * D * 4;
  return SFFN_OK;
}

int sffn_block_norm_backward(const sffn_block_norm* c, const sffn_block_grads* g, void* stream) {
  const int rc = check_call(c);
  if (rc != SFFN_OK) return rc;
  if (!g) return SFFN_ERR_INVALID_ARG;
  const bool channel = c->gate_kind == SFFN_BLOCK_GATE_CHANNEL, full = c->gate_kind == SFFN_BLOCK_GATE_FULL;
  // a gradient of what the call does not have
  if ((c->T > 0 && g->dy && !c->y) || (g->dpost_gain && !c->post_gain) || (g->dpre_gain && !c->pre_gain) || (g->dgate && c->gate_kind == SFFN_BLOCK_GATE_NONE) || (g->dn && !c->pre_gain))
    return SFFN_ERR_INVALID_ARG;
  if (!aligned(g->dpost_gain, 16) || !aligned(g->dpre_gain, 16) || (channel && !aligned(g->dgate, 16)) || !aligned(g->dgate, 4)) return SFFN_ERR_UNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (c->T == 0) {
    float* const columns[3] = {g->dpost_gain, g->dpre_gain, channel ? static_cast<float*>(g->dgate) : nullptr};
    for (float* p : columns)
      if (p) SFFN_CUDA(cudaMemsetAsync(p, 0, (size_t)c->D * 4, s));
    return SFFN_OK;
  }
  if (!g->dy && !g->dresid && !g->dpost_gain && !g->dpre_gain && !g->dgate) return SFFN_OK;
  const size_t ey = element(c->y_dtype), eh = element(c->h_dtype), en = element(c->n_dtype);
  if ((!g->dh && !g->dn) || (g->dn && !c->h) || ((c->post_gain || g->dn) && !c->stats)) return SFFN_ERR_INVALID_ARG;
  int rows = c->y ? check_rows(c->y, c->ld_y, c->D, ey) : SFFN_OK;
  if (rows == SFFN_OK && g->dn) rows = check_rows(c->h, c->ld_h, c->D, eh);
  if (rows == SFFN_OK && g->dh) rows = check_rows(g->dh, g->ld_dh, c->D, eh);
  if (rows == SFFN_OK && g->dn) rows = check_rows(g->dn, g->ld_dn, c->D, en);
  if (rows == SFFN_OK && g->dy) rows = check_rows(g->dy, g->ld_dy, c->D, ey);
  if (rows == SFFN_OK && g->dresid) rows = check_rows(g->dresid, g->ld_dresid, c->D, eh);
  if (rows == SFFN_OK && full && g->dgate) rows = check_rows(g->dgate, g->ld_dgate, c->D, eh);
  if (rows != SFFN_OK) return rows;
  size_t need = 0;
  if (g->dpost_gain || g->dpre_gain || (channel && g->dgate)) {
    sffn_block_norm_workspace_bytes(c->D, &need);
    if (!g->workspace || !aligned(g->workspace, 16) || g->workspace_bytes < need) return SFFN_ERR_WORKSPACE;
  }
  const Span none = {nullptr, 0, 0, 0}, y = rows_of(c->y, c->T, c->D, c->y_dtype, c->ld_y), h = g->dn ? rows_of(c->h, c->T, c->D, c->h_dtype, c->ld_h) : none;
  const Span dh = rows_of(g->dh, c->T, c->D, c->h_dtype, g->ld_dh), dn = rows_of(g->dn, c->T, c->D, c->n_dtype, g->ld_dn);
  const Span dy = rows_of(g->dy, c->T, c->D, c->y_dtype, g->ld_dy), dresid = rows_of(g->dresid, c->T, c->D, c->h_dtype, g->ld_dresid);
  const int64_t columns = 4ll * c->D;
  const Span dpost = whole(g->dpost_gain, columns), dpre = whole(g->dpre_gain, columns), dgate = gate_of(c, g->dgate, g->ld_dgate);
  const Span stats = whole(c->stats, 8ll * c->T), own = need ? whole(g->workspace, (int64_t)need) : none;
  // each row of dresid is written when its row of dh has been read; lines of column sums are written while other rows are still being read
  if (outputs_meet({y, h, dn, stats, gate_of(c, c->gate, c->ld_gate), whole(c->post_gain, columns), whole(c->pre_gain, columns)}, {dy, dresid, dpost, dpre, dgate, own}) ||
      outputs_meet({dh}, {dy, dpost, dpre, dgate, own}) || (meet(dresid, dh) && !same(dresid, dh)))
    return SFFN_ERR_INVALID_ARG;
  int sms = 0;
  const int count = sm_count(&sms);
  if (count != SFFN_OK) return count;
  SFFN_CUDA(sffn::launch_block_backward(*c, *g, static_cast<float*>(need ? g->workspace : nullptr), sms, s));
  return SFFN_OK;
}

}  // extern "C"
