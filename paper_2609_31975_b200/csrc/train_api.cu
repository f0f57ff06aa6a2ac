// Host side of the training calls of the C ABI: argument checks, workspace layout, and the order of the kernels.
#include <algorithm>
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

constexpr double kSplitProducts = 1.5e8;  // T D H
constexpr int kFewForward = 32, kFewBackward = 16;  // tokens
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

// Which kernels serve a call: tensor cores for bf16, and for fp32 from the size on at which splitting every operand into three
// terms and multiplying them six times is faster than fp32 FMAs.  Forward / backward in us, FMAs against terms: T D H = 1.3e8 44 / 89
// against 58 / 80, 1.5e8 64 / 120 against 62 / 107, 2.7e8 78 / 149 against 65 / 91.  Few tokens read the weights once and split them for
// nothing, which a backward pass, with more products, outweighs sooner: 4096 x 8192, 16 tokens 264 / 401 against 349 / 495; 32 tokens forward
// 2048 x 4096 86 against 119, 4096 x 14336 476 against 649; 48 tokens, 3840 x 14230, 968 against 615; backward of 20 tokens there 1224
// against 817.
bool on_tensor_cores(int T, int D, int H, int dtype, bool backward) {
  return dtype == SFFN_BF16 || (T > (backward ? kFewBackward : kFewForward) && (double)T * D * H >= kSplitProducts);
}

struct TrainLayout {
  bool umma, split;         // split: operands in three bf16 terms
  int64_t ld_h, ld_d;       // rows of hidden values, and of the terms of D-wide operands
  int64_t limb_h, limb_t, limb_w;  // elements between the terms of hidden values, of x and dy, of a weight
  size_t partial, h, dz, du, db, x, dy, w[3], total;
  int lines;
};
TrainLayout train_layout(int T, int D, int H, int dtype, bool backward) {
  TrainLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += up256(bytes);
    return o;
  };
  L.umma = on_tensor_cores(T, D, H, dtype, backward);
  L.split = L.umma && dtype == SFFN_F32;
  L.ld_h = hidden_ld(H);
  L.ld_d = hidden_ld(D);
  L.limb_h = T * L.ld_h;
  L.limb_t = T * L.ld_d;
  L.limb_w = H * L.ld_d;
  if (L.umma) {  // what the largest of the call's products may leave in pieces
    const long long of_d = (D + 63) / 64, of_h = (H + 63) / 64, of_t = (T + 63) / 64;
    const size_t room[3] = {sffn::train_umma_partial_bytes(backward ? sffn::kEpiHidden : sffn::kEpiGateUp, L.split, T, H, of_d, 1),
                            sffn::train_umma_partial_bytes(sffn::kEpiStore, L.split, T, D, (backward ? 2 : 1) * of_h, 1),
                            backward ? sffn::train_umma_partial_bytes(sffn::kEpiStore, L.split, H, D, of_t, 3) : 0};
    L.partial = take(std::max({room[0], room[1], room[2]}));
  }
  const size_t hidden = (size_t)T * L.ld_h * (L.split ? 6 : element(dtype));
  L.h = take(hidden);
  L.lines = L.umma ? sffn::train_umma_lines(T) : sffn::train_simt_lines(T);
  if (backward) {
    L.dz = take(hidden);
    L.du = take(hidden);
    L.db = take((size_t)L.lines * L.ld_h * 4);
  }
  if (L.split) {
    L.x = take((size_t)L.limb_t * 6);
    if (backward) L.dy = take((size_t)L.limb_t * 6);
    for (size_t& w : L.w) w = take((size_t)L.limb_w * 6);
  }
  L.total = off > 256 ? off : 256;
  return L;
}

// The products of one call, on the kernels that serve it.
struct Products {
  const sffn_train_call* c;
  TrainLayout L;
  char* ws;
  cudaStream_t s;

  Products(const sffn_train_call* call, bool backward, cudaStream_t stream) : c(call), s(stream) {
    L = train_layout(c->T, c->D, c->H, c->dtype, backward);
    ws = static_cast<char*>(c->workspace);
  }
  void* hidden(size_t at) const { return ws + at; }
  // An operand as the products take it: itself, or its terms, which `at` receives.
  cudaError_t split(const void* in, int64_t ld, int rows, size_t at, int64_t limb) const {
    if (!L.split) return cudaSuccess;
    return sffn::launch_train_split(static_cast<const float*>(in), ld, rows, c->D, reinterpret_cast<__nv_bfloat16*>(ws + at), L.ld_d, limb, s);
  }
  sffn::TrainOperand operand(const void* in, int64_t ld, size_t at) const {
    return L.split ? sffn::TrainOperand{ws + at, L.ld_d} : sffn::TrainOperand{in, ld};
  }
  cudaError_t run(sffn::TrainGemm& g, const int64_t* limb_a, const int64_t* limb_b, int* lines = nullptr) const {
    int unused = 0;
    g.epi.limb = L.limb_h;
    if (!g.a_major_k && !L.split && g.K <= (c->dtype == SFFN_BF16 ? sffn::kOuterBf16 : sffn::kOuterF32)) return sffn::launch_train_outer(g, c->dtype, s);
    if (!L.umma) return sffn::launch_train_simt(g, lines ? lines : &unused, s);
    if (lines) *lines = L.lines;
    sffn::TrainUmma t{};
    t.g = g;
    t.f32 = L.split;
    for (int i = 0; i < 3; ++i) {
      t.limb_a[i] = limb_a[i];
      t.limb_b[i] = limb_b[i];
    }
    t.partial = reinterpret_cast<float*>(ws + L.partial);
    t.status = c->status;
    return sffn::launch_train_umma(t, s);
  }
};

int check_shape(int T, int D, int H, int dtype) {
  if (T < 0 || D <= 0 || H <= 0 || !storage_type(dtype)) return SFFN_ERR_INVALID_ARG;
  if ((D * element(dtype)) % 16 || T > kMaxRows || H > kMaxRows || D > kMaxRows) return SFFN_ERR_UNSUPPORTED;
  return SFFN_OK;
}

int check_rows(const void* p, int64_t ld, int64_t width, size_t esz) {
  if (ld < width) return SFFN_ERR_INVALID_ARG;
  return aligned(p, 16) && (ld * esz) % 16 == 0 && ld <= (1ll << 31) ? SFFN_OK : SFFN_ERR_UNSUPPORTED;
}

// A matrix's rows in memory, and whether any of them meets any row of another matrix's (what lies between rows does not count: two
// matrices may be columns of one).
struct Span {
  const void* p;
  int64_t rows, width, ld;  // bytes
};
bool meet(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0 || a.width <= 0 || b.width <= 0) return false;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));  // b's first byte, from a's
  if (d >= (a.rows - 1) * a.ld + a.width || -d >= (b.rows - 1) * b.ld + b.width) return false;
  if (a.ld == b.ld) {  // rows i of a and j of b meet where d - a.width < (i - j) ld < d + b.width
    const auto below = [](int64_t v, int64_t n) { return v >= 0 ? v / n : -((-v + n - 1) / n); };
    const int64_t least = below(d - a.width, a.ld) + 1, most = -below(-(d + b.width), a.ld) - 1;
    return (least > 1 - b.rows ? least : 1 - b.rows) <= (most < a.rows - 1 ? most : a.rows - 1);
  }
  for (int64_t i = 0, j = 0; i < a.rows && j < b.rows;) {
    if (i * a.ld + a.width <= d + j * b.ld) ++i;
    else if (d + j * b.ld + b.width <= i * a.ld) ++j;
    else return true;
  }
  return false;
}
// Whether an output of a call meets one of these inputs, or another output.
template <size_t kIn, size_t kOut>
bool outputs_meet(const Span (&in)[kIn], const Span (&out)[kOut]) {
  for (size_t o = 0; o < kOut; ++o) {
    for (const Span& i : in)
      if (meet(out[o], i)) return true;
    for (size_t q = o + 1; q < kOut; ++q)
      if (meet(out[o], out[q])) return true;
  }
  return false;
}
Span whole(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }

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
  const Products p(c, false, static_cast<cudaStream_t>(stream));
  const TrainLayout& L = p.L;
  const int64_t esz = (int64_t)element(c->dtype), matrix = esz * c->H * c->D;
  const Span x = {c->x, c->T, esz * c->D, esz * c->ld_x}, own = whole(c->workspace, (int64_t)L.total);
  const Span out = {y, c->T, esz * c->D, esz * ld_y}, z = {c->z, c->T, esz * c->H, esz * c->ld_hidden}, u = {c->u, c->T, esz * c->H, esz * c->ld_hidden};
  const Span W[3] = {whole(c->W_g, matrix), whole(c->W_up, matrix), whole(c->W_down, matrix)}, bias = whole(c->b_g, 4ll * c->H);
  // y is written when x has been read for the last time
  if (outputs_meet({W[0], W[1], W[2], bias, own}, {out, z, u}) || meet(x, z) || meet(x, u)) return SFFN_ERR_INVALID_ARG;
  const int64_t tokens[3] = {L.limb_t, L.limb_t, L.limb_t}, weights[3] = {L.limb_w, L.limb_w, L.limb_w}, hidden[3] = {L.limb_h, L.limb_h, L.limb_h};
  SFFN_CUDA(p.split(c->x, c->ld_x, c->T, L.x, L.limb_t));
  SFFN_CUDA(p.split(c->W_g, c->D, c->H, L.w[0], L.limb_w));
  SFFN_CUDA(p.split(c->W_up, c->D, c->H, L.w[1], L.limb_w));
  SFFN_CUDA(p.split(c->W_down, c->D, c->H, L.w[2], L.limb_w));

  sffn::TrainGemm up{};
  up.M = c->T; up.N = c->H; up.K = c->D;
  up.parts = 2; up.batch = 1;
  up.a[0] = p.operand(c->x, c->ld_x, L.x);
  up.b[0] = p.operand(c->W_g, c->D, L.w[0]);
  up.b[1] = p.operand(c->W_up, c->D, L.w[1]);
  up.a_major_k = up.b_major_k = true;
  up.epilogue = sffn::kEpiGateUp;
  sffn::TrainEpilogue& e = up.epi;
  e.M = c->T; e.N = c->H; e.act = c->act; e.act_up = c->act_up;
  e.bias = c->b_g; e.z = c->z; e.u = c->u; e.ld_zu = c->ld_hidden;
  e.h = p.hidden(L.h); e.ld_h = L.ld_h;
  SFFN_CUDA(p.run(up, tokens, weights));

  sffn::TrainGemm down{};
  down.M = c->T; down.N = c->D; down.K = c->H;
  down.parts = down.batch = 1;
  down.a[0] = {p.hidden(L.h), L.ld_h};
  down.b[0] = p.operand(c->W_down, c->D, L.w[2]);
  down.a_major_k = true; down.b_major_k = false;
  down.epilogue = sffn::kEpiStore;
  down.epi.M = c->T; down.epi.N = c->D;
  down.epi.out[0] = y; down.epi.ld_out = ld_y;
  SFFN_CUDA(p.run(down, hidden, weights));
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
  const Products p(c, true, s);
  const TrainLayout& L = p.L;
  const bool want_dz = g->dx || g->dW_g, want_du = g->dx || g->dW_up, want_dh = want_dz || want_du || g->db_g;
  if (!want_dh && !g->dW_down) return SFFN_OK;
  {
    const int64_t e = (int64_t)esz, T = c->T, D = c->D, H = c->H, matrix = e * H * D;
    const Span x = {c->x, T, e * D, e * c->ld_x}, dys = {dy, T, e * D, e * ld_dy}, z = {c->z, T, e * H, e * c->ld_hidden}, u = {c->u, T, e * H, e * c->ld_hidden};
    const Span W[3] = {whole(c->W_g, matrix), whole(c->W_up, matrix), whole(c->W_down, matrix)}, own = whole(c->workspace, (int64_t)L.total);
    const Span dx = {g->dx, T, e * D, e * g->ld_dx}, w[3] = {whole(g->dW_g, matrix), whole(g->dW_up, matrix), whole(g->dW_down, matrix)};
    const Span db = whole(g->db_g, 4 * H);
    // dx is written last: what it may lie over has been read by then
    if (outputs_meet({W[0], W[1], W[2], own}, {dx, w[0], w[1], w[2], db}) || outputs_meet({x, dys, z, u}, {w[0], w[1], w[2], db})) return SFFN_ERR_INVALID_ARG;
  }
  const int64_t tokens[3] = {L.limb_t, L.limb_t, L.limb_t}, weights[3] = {L.limb_w, L.limb_w, L.limb_w}, hidden[3] = {L.limb_h, L.limb_h, L.limb_h};
  void* const values[3] = {p.hidden(L.dz), p.hidden(L.du), p.hidden(L.h)};
  float* const lines = reinterpret_cast<float*>(p.ws + L.db);
  SFFN_CUDA(p.split(dy, ld_dy, c->T, L.dy, L.limb_t));
  SFFN_CUDA(p.split(c->W_down, c->D, c->H, L.w[2], L.limb_w));
  if (g->dW_g || g->dW_up) SFFN_CUDA(p.split(c->x, c->ld_x, c->T, L.x, L.limb_t));
  if (g->dx) {
    SFFN_CUDA(p.split(c->W_g, c->D, c->H, L.w[0], L.limb_w));
    SFFN_CUDA(p.split(c->W_up, c->D, c->H, L.w[1], L.limb_w));
  }

  sffn::TrainGemm dh{};
  dh.M = c->T; dh.N = c->H; dh.K = c->D;
  dh.parts = dh.batch = 1;
  dh.a[0] = p.operand(dy, ld_dy, L.dy);
  dh.b[0] = p.operand(c->W_down, c->D, L.w[2]);
  dh.a_major_k = dh.b_major_k = true;
  dh.epilogue = sffn::kEpiHidden;
  sffn::TrainEpilogue& e = dh.epi;
  e.M = c->T; e.N = c->H; e.act = c->act; e.act_up = c->act_up;
  e.z = c->z; e.u = c->u; e.ld_zu = c->ld_hidden; e.ld_h = L.ld_h;
  e.dz = want_dz ? values[0] : nullptr;
  e.du = want_du ? values[1] : nullptr;
  e.h = g->dW_down ? values[2] : nullptr;
  e.db = g->db_g ? lines : nullptr;
  int n_lines = 0;
  SFFN_CUDA(p.run(dh, tokens, weights, &n_lines));
  if (g->db_g) SFFN_CUDA(sffn::launch_train_column_sums(lines, n_lines, L.ld_h, c->H, g->db_g, s));

  sffn::TrainGemm dw{};
  dw.M = c->H; dw.N = c->D; dw.K = c->T;
  dw.parts = 1;
  for (int i = 0; i < 3; ++i) {
    if (!dW[i]) continue;
    dw.a[dw.batch] = {values[i], L.ld_h};
    dw.b[dw.batch] = i < 2 ? p.operand(c->x, c->ld_x, L.x) : p.operand(dy, ld_dy, L.dy);
    dw.epi.out[dw.batch++] = dW[i];
  }
  dw.a_major_k = dw.b_major_k = false;
  dw.epilogue = sffn::kEpiStore;
  dw.epi.M = c->H; dw.epi.N = c->D; dw.epi.ld_out = c->D;
  if (dw.batch > 0) SFFN_CUDA(p.run(dw, hidden, tokens));

  if (g->dx) {
    sffn::TrainGemm dx{};
    dx.M = c->T; dx.N = c->D; dx.K = c->H;
    dx.parts = 2; dx.batch = 1;
    dx.a[0] = {values[0], L.ld_h};
    dx.a[1] = {values[1], L.ld_h};
    dx.b[0] = p.operand(c->W_g, c->D, L.w[0]);
    dx.b[1] = p.operand(c->W_up, c->D, L.w[1]);
    dx.a_major_k = true; dx.b_major_k = false;
    dx.epilogue = sffn::kEpiStore;
    dx.epi.M = c->T; dx.epi.N = c->D;
    dx.epi.out[0] = g->dx; dx.epi.ld_out = g->ld_dx;
    SFFN_CUDA(p.run(dx, hidden, weights));
  }
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
  // 2^-50 is the root of the largest v that codes hold as zero: with a smaller eps there would be next to nothing to divide by
  for (int i = 0; i < n; ++i)
    if (t[i].state_bits == 8 && c->eps < 0x1p-50) return SFFN_ERR_UNSUPPORTED;
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
