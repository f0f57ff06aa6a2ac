// Host side of the training calls of the C ABI: argument checks, workspace layout, and the order of the kernels.
#include <cmath>

#include "optim_kernels.cuh"
#include "sparse_ffn.h"
#include "train_kernels.cuh"

namespace sffn {
void note_cuda_error(cudaError_t e, const char* file, int line);  // api.cu
}

namespace {

#define SFFN_CUDA(expr)                                   \
  do {                                                    \
    const cudaError_t e_ = (expr);                        \
    if (e_ != cudaSuccess) {                              \
      sffn::note_cuda_error(e_, "train_api.cu", __LINE__); \
      return SFFN_ERR_CUDA;                               \
    }                                                     \
  } while (0)

constexpr int kMaxRows = 1 << 22;  // tokens, and neurons: the kernels' grids and tensor maps have room for so many

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline size_t element(int dtype) { return dtype == SFFN_BF16 ? 2 : 4; }
inline int64_t hidden_ld(int H) { return ((int64_t)H + 7) / 8 * 8; }
inline bool storage_type(int dtype) { return dtype == SFFN_F32 || dtype == SFFN_BF16; }
inline bool any_act(int act) { return act >= SFFN_ACT_RELU && act <= SFFN_ACT_SILU; }

int sm_count(int* n) {
  int dev = 0;
  SFFN_CUDA(cudaGetDevice(&dev));
  SFFN_CUDA(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
  return SFFN_OK;
}

struct TrainLayout {
  size_t h, dz, du, db, total;
};
TrainLayout train_layout(int T, int D, int H, int dtype, bool backward) {
  TrainLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += up256(bytes);
    return o;
  };
  const size_t hidden = (size_t)T * hidden_ld(H) * element(dtype);
  L.h = take(hidden);
  if (backward) {
    L.dz = take(hidden);
    L.du = take(hidden);
    L.db = take((size_t)sffn::train_simt_lines(T) * hidden_ld(H) * 4);
  }
  L.total = off > 256 ? off : 256;
  return L;
}

int check_shape(int T, int D, int H, int dtype) {
  if (T < 0 || D <= 0 || H <= 0 || !storage_type(dtype)) return SFFN_ERR_INVALID_ARG;
  if ((D * element(dtype)) % 16 || T > kMaxRows || H > kMaxRows || D > kMaxRows) return SFFN_ERR_UNSUPPORTED;
  return SFFN_OK;
}

int check_rows(const void* p, int64_t ld, int64_t width, size_t esz) {
  if (ld < width) return SFFN_ERR_INVALID_ARG;
  return aligned(p, 16) && (ld * esz) % 16 == 0 && ld <= (1ll << 31) ? SFFN_OK : SFFN_ERR_UNSUPPORTED;
}

int check_call(const sffn_train_call* c, bool backward) {
  if (!c) return SFFN_ERR_INVALID_ARG;
  const int shape = check_shape(c->T, c->D, c->H, c->dtype);
  if (shape != SFFN_OK) return shape;
  if (!any_act(c->act) || !any_act(c->act_up) || !c->status) return SFFN_ERR_INVALID_ARG;
  const size_t esz = element(c->dtype);
  if (!c->W_g || !c->W_up || !c->W_down) return SFFN_ERR_INVALID_ARG;
  if (!aligned(c->W_g, 16) || !aligned(c->W_up, 16) || !aligned(c->W_down, 16) || !aligned(c->b_g, 4) || !aligned(c->status, 4)) return SFFN_ERR_UNSUPPORTED;
  if (c->T > 0) {
    if (!c->x) return SFFN_ERR_INVALID_ARG;
    int rows = check_rows(c->x, c->ld_x, c->D, esz);
    if (rows != SFFN_OK) return rows;
    if (!c->z != !c->u || (backward && !c->z)) return SFFN_ERR_INVALID_ARG;
    if (c->z) {
      rows = check_rows(c->z, c->ld_hidden, c->H, esz);
      if (rows != SFFN_OK) return rows;
      if (!aligned(c->u, 16)) return SFFN_ERR_UNSUPPORTED;
    }
  }
  size_t need = 0;
  const int rc = sffn_train_workspace_bytes(c->T, c->D, c->H, c->dtype, backward, &need);
  if (rc != SFFN_OK) return rc;
  return c->workspace && aligned(c->workspace, 256) && c->workspace_bytes >= need ? SFFN_OK : SFFN_ERR_WORKSPACE;
}

}  // namespace

extern "C" {

int sffn_train_workspace_bytes(int T, int D, int H, int dtype, int backward, size_t* bytes) {
  if (!bytes) return SFFN_ERR_INVALID_ARG;
  const int shape = check_shape(T, D, H, dtype);
  if (shape != SFFN_OK) return shape;
  *bytes = train_layout(T, D, H, dtype, backward != 0).total;
  return SFFN_OK;
}

int gated_ffn_forward(const sffn_train_call* c, void* y, int64_t ld_y, void* stream) {
  int rc = check_call(c, false);
  if (rc != SFFN_OK) return rc;
  if (c->T == 0) return SFFN_OK;
  if (!y) return SFFN_ERR_INVALID_ARG;
  rc = check_rows(y, ld_y, c->D, element(c->dtype));
  if (rc != SFFN_OK) return rc;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(c->workspace);
  const TrainLayout L = train_layout(c->T, c->D, c->H, c->dtype, false);
  const int64_t ld_h = hidden_ld(c->H);

  sffn::TrainGemm up{};
  up.M = c->T; up.N = c->H; up.K = c->D;
  up.parts = 2; up.batch = 1;
  up.a[0] = {c->x, c->ld_x};
  up.b[0] = {c->W_g, c->D};
  up.b[1] = {c->W_up, c->D};
  up.a_major_k = up.b_major_k = true;
  up.epilogue = sffn::kEpiGateUp;
  sffn::TrainEpilogue& e = up.epi;
  e.M = c->T; e.N = c->H; e.act = c->act; e.act_up = c->act_up;
  e.bias = c->b_g; e.z = c->z; e.u = c->u; e.ld_zu = c->ld_hidden;
  e.h = ws + L.h; e.ld_h = ld_h;
  SFFN_CUDA(sffn::launch_train_simt(up, c->dtype, s));

  sffn::TrainGemm down{};
  down.M = c->T; down.N = c->D; down.K = c->H;
  down.parts = down.batch = 1;
  down.a[0] = {ws + L.h, ld_h};
  down.b[0] = {c->W_down, c->D};
  down.a_major_k = true; down.b_major_k = false;
  down.epilogue = sffn::kEpiStore;
  down.epi.M = c->T; down.epi.N = c->D;
  down.epi.out[0] = y; down.epi.ld_out = ld_y;
  SFFN_CUDA(sffn::launch_train_simt(down, c->dtype, s));
  return SFFN_OK;
}

int gated_ffn_backward(const sffn_train_call* c, const void* dy, int64_t ld_dy, const sffn_train_grads* g, void* stream) {
  int rc = check_call(c, true);
  if (rc != SFFN_OK) return rc;
  if (!g) return SFFN_ERR_INVALID_ARG;
  const size_t esz = element(c->dtype);
  if (!aligned(g->dW_g, 16) || !aligned(g->dW_up, 16) || !aligned(g->dW_down, 16) || !aligned(g->db_g, 4)) return SFFN_ERR_UNSUPPORTED;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  void* const dW[3] = {g->dW_g, g->dW_up, g->dW_down};
  if (c->T == 0) {
    for (void* w : dW)
      if (w) SFFN_CUDA(cudaMemsetAsync(w, 0, (size_t)c->H * c->D * esz, s));
    if (g->db_g) SFFN_CUDA(cudaMemsetAsync(g->db_g, 0, (size_t)c->H * 4, s));
    return SFFN_OK;
  }
  if (!dy) return SFFN_ERR_INVALID_ARG;
  rc = check_rows(dy, ld_dy, c->D, esz);
  if (rc != SFFN_OK) return rc;
  if (g->dx) {
    rc = check_rows(g->dx, g->ld_dx, c->D, esz);
    if (rc != SFFN_OK) return rc;
  }
  char* ws = static_cast<char*>(c->workspace);
  const TrainLayout L = train_layout(c->T, c->D, c->H, c->dtype, true);
  const int64_t ld_h = hidden_ld(c->H);
  void* const hidden[3] = {ws + L.dz, ws + L.du, ws + L.h};
  float* const lines = reinterpret_cast<float*>(ws + L.db);

  sffn::TrainGemm dh{};
  dh.M = c->T; dh.N = c->H; dh.K = c->D;
  dh.parts = dh.batch = 1;
  dh.a[0] = {dy, ld_dy};
  dh.b[0] = {c->W_down, c->D};
  dh.a_major_k = dh.b_major_k = true;
  dh.epilogue = sffn::kEpiHidden;
  sffn::TrainEpilogue& e = dh.epi;
  e.M = c->T; e.N = c->H; e.act = c->act; e.act_up = c->act_up;
  e.z = c->z; e.u = c->u; e.ld_zu = c->ld_hidden; e.ld_h = ld_h;
  e.dz = g->dx || g->dW_g ? hidden[0] : nullptr;
  e.du = g->dx || g->dW_up ? hidden[1] : nullptr;
  e.h = g->dW_down ? hidden[2] : nullptr;
  e.db = g->db_g ? lines : nullptr;
  if (e.dz || e.du || e.h || e.db) SFFN_CUDA(sffn::launch_train_simt(dh, c->dtype, s));
  if (g->db_g) SFFN_CUDA(sffn::launch_train_column_sums(lines, sffn::train_simt_lines(c->T), ld_h, c->H, g->db_g, s));

  if (g->dx) {
    sffn::TrainGemm dx{};
    dx.M = c->T; dx.N = c->D; dx.K = c->H;
    dx.parts = 2; dx.batch = 1;
    dx.a[0] = {hidden[0], ld_h};
    dx.a[1] = {hidden[1], ld_h};
    dx.b[0] = {c->W_g, c->D};
    dx.b[1] = {c->W_up, c->D};
    dx.a_major_k = true; dx.b_major_k = false;
    dx.epilogue = sffn::kEpiStore;
    dx.epi.M = c->T; dx.epi.N = c->D;
    dx.epi.out[0] = g->dx; dx.epi.ld_out = g->ld_dx;
    SFFN_CUDA(sffn::launch_train_simt(dx, c->dtype, s));
  }
  sffn::TrainGemm dw{};
  dw.M = c->H; dw.N = c->D; dw.K = c->T;
  dw.parts = 1;
  for (int i = 0; i < 3; ++i) {
    if (!dW[i]) continue;
    dw.a[dw.batch] = {hidden[i], ld_h};
    dw.b[dw.batch] = i < 2 ? sffn::TrainOperand{c->x, c->ld_x} : sffn::TrainOperand{dy, ld_dy};
    dw.epi.out[dw.batch++] = dW[i];
  }
  if (dw.batch == 0) return SFFN_OK;
  dw.a_major_k = dw.b_major_k = false;
  dw.epilogue = sffn::kEpiStore;
  dw.epi.M = c->H; dw.epi.N = c->D; dw.epi.ld_out = c->D;
  SFFN_CUDA(sffn::launch_train_simt(dw, c->dtype, s));
  return SFFN_OK;
}

int sffn_grad_norm(const sffn_tensor* t, int n, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (n < 0 || (n > 0 && !t) || !norm) return SFFN_ERR_INVALID_ARG;
  if (!aligned(norm, 4)) return SFFN_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < SFFN_GRAD_NORM_WORKSPACE) return SFFN_ERR_WORKSPACE;
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0 || (t[i].n > 0 && !t[i].data) || !storage_type(t[i].dtype)) return SFFN_ERR_INVALID_ARG;
    if (t[i].n > (1ll << 38) || !aligned(t[i].data, element(t[i].dtype))) return SFFN_ERR_UNSUPPORTED;
  }
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != SFFN_OK) return rc;
  SFFN_CUDA(sffn::launch_grad_norm(t, n, norm, workspace, sms, static_cast<cudaStream_t>(stream)));
  return SFFN_OK;
}

static int check_states(const sffn_adamw_tensor* t, int n, bool step) {
  if (n < 0 || (n > 0 && !t)) return SFFN_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const sffn_adamw_tensor& a = t[i];
    if (a.n < 0 || (a.state_bits != 8 && a.state_bits != 32)) return SFFN_ERR_INVALID_ARG;
    if (a.n > (1ll << 38)) return SFFN_ERR_UNSUPPORTED;
    if (step) {
      if (!storage_type(a.p_dtype) || !storage_type(a.g_dtype) || (a.master && a.p_dtype != SFFN_BF16)) return SFFN_ERR_INVALID_ARG;
      if (!std::isfinite(a.lr) || !std::isfinite(a.weight_decay)) return SFFN_ERR_INVALID_ARG;
    } else if (a.state_bits != 8) {
      return SFFN_ERR_INVALID_ARG;
    }
    if (a.n == 0) continue;
    if (!a.m || !a.v || (step && (!a.p || !a.g)) || (a.state_bits == 8 && (!a.m_scale || !a.v_scale))) return SFFN_ERR_INVALID_ARG;
    if (step && (!aligned(a.p, element(a.p_dtype)) || !aligned(a.g, element(a.g_dtype)) || !aligned(a.master, 4))) return SFFN_ERR_UNSUPPORTED;
    if (a.state_bits == 8 ? !aligned(a.m_scale, 4) || !aligned(a.v_scale, 4) : !aligned(a.m, 4) || !aligned(a.v, 4)) return SFFN_ERR_UNSUPPORTED;
  }
  return SFFN_OK;
}

int sffn_adamw_step(const sffn_adamw_tensor* t, int n, const sffn_adamw_config* c, void* stream) {
  int rc = check_states(t, n, true);
  if (rc != SFFN_OK) return rc;
  if (!c || c->step < 1 || !(c->beta1 >= 0 && c->beta1 < 1) || !(c->beta2 >= 0 && c->beta2 < 1) || !(c->eps >= 0) || std::isinf(c->eps)) return SFFN_ERR_INVALID_ARG;
  if (c->grad_norm && !(c->max_norm > 0)) return SFFN_ERR_INVALID_ARG;
  if (!aligned(c->grad_norm, 4)) return SFFN_ERR_UNSUPPORTED;
  int sms = 0;
  rc = sm_count(&sms);
  if (rc != SFFN_OK) return rc;
  SFFN_CUDA(sffn::launch_adamw(t, n, *c, sms, static_cast<cudaStream_t>(stream)));
  return SFFN_OK;
}

int sffn_adamw_state_values(const sffn_adamw_tensor* t, int n, float* const* m_out, float* const* v_out, void* stream) {
  int rc = check_states(t, n, false);
  if (rc != SFFN_OK) return rc;
  for (int i = 0; i < n; ++i)
    if ((m_out && !aligned(m_out[i], 4)) || (v_out && !aligned(v_out[i], 4))) return SFFN_ERR_UNSUPPORTED;
  int sms = 0;
  rc = sm_count(&sms);
  if (rc != SFFN_OK) return rc;
  SFFN_CUDA(sffn::launch_adamw_values(t, n, m_out, v_out, sms, static_cast<cudaStream_t>(stream)));
  return SFFN_OK;
}

}  // extern "C"
