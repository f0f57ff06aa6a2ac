// Host side of the orthogonalised update and the Muon step: argument checks, batches of matrices of one shape, workspace layout, the order of
// the kernels, and the powers of two that everything in sixteen bits is stored with.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#define SFFN_FILE "muon_api.cu"
#include "host_checks.cuh"
#include "muon_kernels.cuh"
#include "sparse_ffn.h"

using namespace sffn::host;
using sffn::MuonBatch;
using sffn::MuonItem;

namespace {

constexpr int kMaxShort = 1 << 16, kMaxLong = 1 << 22;  // sides of a matrix: tiles' numbers and tensor maps have room for so many
// Entries of a batch, but for a matrix that has more by itself: matrices of which one fills the device take turns in one workspace.
constexpr int64_t kBatchEntries = 1ll << 26;
constexpr double kLargestBound = 1 << 30;

struct Matrix {
  MuonItem item;
  int R, C;
  bool src_bf16, out_bf16;
  int terms;
};

// ---- powers of two ----------------------------------------------------------------------------------------------------
// A matrix whose singular values are at most `bound` is stored with 2^e: entries stay below 2^14, a quarter of what fp16 holds.
int exponent(double bound) { return sffn::kMuonExponent - (int)std::ceil(std::log2(std::max(bound, 0x1p-20))); }


// What a call launches for every batch (muon_umma.cu has the forms).  Singular values are followed at 2049 points of what they can be, with
// 2 % for what lies between and for roundings: what X and the polynomials of A reach gives the powers of two.
using Products = std::vector<sffn::MuonProduct>;
constexpr int kPoints = 2049;
double most(const std::vector<double>& v) {
  double m = 0;
  for (double x : v) m = std::max(m, std::fabs(x));
  return 1.02 * m;
}

// `group` steps at a time.  false: coefficients under which singular values leave every bound.
bool make_products(const sffn_newton_schulz& ns, int group, Products& out) {
  using sffn::MuonTerm;
  struct Held {  // a matrix: where, with which exponent
    int which, e;
  };
  const MuonTerm none = {-1, 0, 0.f, -1};
  auto with = [](const Held& h, double c, int factor) { return MuonTerm{h.which, h.e, (float)c, factor}; };
  auto only = [](double c, int factor) { return MuonTerm{-1, 0, (float)c, factor}; };
  double bound = 1.0;  // of X's singular values: the first X has norm 1
  for (int k = 0, from = 0; k < ns.steps; from ^= 1) {
    const int steps = std::min(group, ns.steps - k), ex = exponent(bound);
    const bool first = k == 0;
    // The first X is stored up to a factor 1 < g <= 2 smaller than it is: A's entries are smaller for it, those with a factor g larger.
    const double g = first ? 2.0 : 1.0;
    auto factor = [&](int which) { return first ? which : -1; };  // of g: its first, second, third and fifth power
    std::vector<double> x(kPoints), poly(kPoints), rest(kPoints), now(kPoints);  // singular values, what B, R and a result have for them
    for (int i = 0; i < kPoints; ++i) x[i] = bound * i / (kPoints - 1);
    bool bounded = true;
    auto result = [&](int which, double scale) {
      const double m = scale * most(now);
      bounded = bounded && m <= kLargestBound;
      return Held{which, exponent(m)};
    };
    auto push = [&](int kind, const Held& r, MuonTerm m, MuonTerm n, MuonTerm coefficient) {
      out.push_back({kind, from, r.which, first, m, n, coefficient, ex, r.e, false});
    };
    for (int i = 0; i < kPoints; ++i) now[i] = x[i] * x[i];
    Held A = result(0, 1.0), B{}, R{};
    push(sffn::kGram, A, none, none, none);
    double q = 0;
    for (int j = 0; j < steps; ++j) {
      const double *const c = ns.coefficients + 3 * (k + j), *const before = c - 3;
      for (int i = 0; i < 3; ++i)
        if (!std::isfinite(c[i])) return false;
      const bool scaled = first && j == 0, was = first && j == 1;  // the coefficients of the very first step come with powers of g
      if (j > 0) {  // A of the step before to this one's: D = a A + A B, A = a D + D B
        for (int i = 0; i < kPoints; ++i) now[i] = x[i] * x[i] * (before[0] + poly[i]);
        const int free = 6 - A.which - B.which - R.which;
        const Held D = result(j == 1 ? 2 : free, 1.0);
        push(sffn::kForm, D, with(A, before[0], was ? 0 : -1), with(B, 0, -1), only(1, -1));
        for (int i = 0; i < kPoints; ++i) {
          x[i] *= before[0] + poly[i];
          now[i] = x[i] * x[i];
        }
        A = result(A.which, 1.0);
        push(sffn::kForm, A, with(D, before[0], was ? 0 : -1), with(B, 0, -1), only(1, -1));
        for (int i = 0; i < kPoints; ++i) now[i] = poly[i] = x[i] * x[i] * (c[1] + x[i] * x[i] * c[2]);
        B = result(D.which, 1.0);
      } else {
        for (int i = 0; i < kPoints; ++i) now[i] = poly[i] = x[i] * x[i] * (c[1] + x[i] * x[i] * c[2]);
        B = result(1, g);
      }
      push(sffn::kForm, B, with(A, c[1], scaled ? 2 : -1), with(A, 0, -1), only(c[2], scaled ? 3 : -1));
      if (j == 0) {
        R = B;
        rest = poly;
        q = c[0];
      } else {  // R = q B + a R + R B
        for (int i = 0; i < kPoints; ++i) now[i] = rest[i] = q * poly[i] + c[0] * rest[i] + rest[i] * poly[i];
        const Held last = R;
        R = result(6 - A.which - B.which - R.which, g);
        push(sffn::kForm, R, with(last, c[0], -1), with(B, q, factor(0)), only(1, -1));
        q *= c[0];
      }
    }
    const double* const c = ns.coefficients + 3 * (k + steps - 1);
    for (int i = 0; i < kPoints; ++i) now[i] = x[i] *= c[0] + poly[i];
    bound = most(now);
    k += steps;
    const bool last = k == ns.steps;
    push(last ? sffn::kLast : sffn::kApply, Held{0, last ? 0 : exponent(bound)}, with(R, 0, -1), none, only(q, factor(0)));
    double growth = 1;
    for (int i = k; i < ns.steps; ++i) growth *= std::fabs(ns.coefficients[3 * i]);
    out.back().late = growth <= 4;
    if (!bounded || !(bound <= kLargestBound)) return false;
  }
  return true;
}

// Steps at a time: one, two, three.  Where the longer side of X is longer than the shorter one, a step in the company of others is four products
// of S x S instead of two, and saves a Gram matrix and a product with X.  Roundings in between are not made good again by the next Gram
// matrix, and grow: in 16 bits two steps are within a third of what one by one are off (2048 x 1024 6.2e-4 and 4.7e-4), a factor of two where
// singular values are far apart, three are not; with operands in two terms three are (2^-11 of the errors).
struct Plans {
  Products of[3];
};
// What follows from coefficients alone takes half a millisecond: a thread keeps what its last ones gave.
int check_ns(const sffn_newton_schulz* ns, const Plans** plans) {
  if (!ns || ns->steps < 1 || ns->steps > SFFN_NS_MAX_STEPS || !ns->coefficients || !(ns->eps >= 0) || std::isinf(ns->eps)) return SFFN_ERR_INVALID_ARG;
  if (ns->bits != 0 && ns->bits != 16 && ns->bits != 32) return SFFN_ERR_INVALID_ARG;
  struct Last {
    std::vector<double> coefficients;
    Plans plans;
  };
  static thread_local Last last;
  const size_t n = (size_t)3 * ns->steps;
  if (last.coefficients.size() != n || std::memcmp(last.coefficients.data(), ns->coefficients, n * sizeof(double)) != 0) {
    last.coefficients.clear();  // (until the plans are there)
    for (int i = 0; i < 3; ++i) {
      last.plans.of[i].clear();
      if (!make_products(*ns, i + 1, last.plans.of[i])) return SFFN_ERR_INVALID_ARG;
    }
    last.coefficients.assign(ns->coefficients, ns->coefficients + n);
  }
  *plans = &last.plans;
  return SFFN_OK;
}

int check_shape(int rows, int cols) {
  if (rows < 0 || cols < 0) return SFFN_ERR_INVALID_ARG;
  return std::min(rows, cols) > kMaxShort || std::max(rows, cols) > kMaxLong ? SFFN_ERR_UNSUPPORTED : SFFN_OK;
}

// ---- batches ----------------------------------------------------------------------------------------------------------

// Matrices of one shape and kind, in the order that the caller has them, as many at a time as a batch takes.
std::vector<std::vector<const Matrix*>> batches_of(const std::vector<Matrix>& all) {
  std::vector<const Matrix*> left;
  for (const Matrix& m : all)
    if (m.R > 0 && m.C > 0) left.push_back(&m);
  std::stable_sort(left.begin(), left.end(), [](const Matrix* a, const Matrix* b) {
    const int64_t x[5] = {a->R, a->C, a->src_bf16, a->out_bf16, a->terms}, y[5] = {b->R, b->C, b->src_bf16, b->out_bf16, b->terms};
    return std::lexicographical_compare(x, x + 5, y, y + 5);
  });
  std::vector<std::vector<const Matrix*>> out;
  for (const Matrix* m : left) {
    const bool joins = !out.empty() && [&] {
      const Matrix* f = out.back()[0];
      const int64_t with = (int64_t)out.back().size() + 1;
      return f->R == m->R && f->C == m->C && f->src_bf16 == m->src_bf16 && f->out_bf16 == m->out_bf16 && f->terms == m->terms && with <= sffn::kMuonBatch &&
             with * m->R * m->C <= kBatchEntries;
    }();
    if (!joins) out.emplace_back();
    out.back().push_back(m);
  }
  return out;
}

// The workspace of a batch; `base` NULL: only its size.
size_t layout(MuonBatch& b, int n, const Matrix& like, char* base) {
  b.n = n;
  b.R = like.R; b.C = like.C;
  b.tall = like.R > like.C;
  b.S = std::min(like.R, like.C);
  b.L = std::max(like.R, like.C);
  b.src_bf16 = like.src_bf16;
  b.out_bf16 = like.out_bf16;
  b.terms = like.terms;
  b.ld_x = ((int64_t)b.C + 15) / 16 * 16;
  b.ld_p = ((int64_t)b.S + 15) / 16 * 16;
  b.x_matrix = b.R * b.ld_x;
  b.p_matrix = b.S * b.ld_p;
  b.x_term = n * b.x_matrix;
  b.p_term = n * b.p_matrix;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* const at = base + off;
    off += up256(bytes);
    return base ? at : nullptr;
  };
  for (uint16_t*& x : b.x) x = reinterpret_cast<uint16_t*>(take((size_t)b.x_term * 4));
  for (uint16_t*& m : b.sym) m = reinterpret_cast<uint16_t*>(take((size_t)b.p_term * 2 * b.terms));
  b.diag = reinterpret_cast<float*>(take((size_t)4 * n * ((b.S + 15) / 16 * 16) * 4));
  b.first = reinterpret_cast<float*>(take((size_t)n * 16));
  b.squares = reinterpret_cast<double*>(take((size_t)n * sffn::kMuonPartials * 8));
  b.partial = reinterpret_cast<float*>(take(sffn::muon_partial_floats(b.S, b.R, b.C, n, b.terms) * 4));
  return off;
}

size_t workspace_of(const std::vector<Matrix>& all) {
  size_t need = 256;
  for (const auto& batch : batches_of(all)) {
    MuonBatch b{};
    need = std::max(need, layout(b, (int)batch.size(), *batch[0], nullptr));
  }
  return need;
}

// Everything that a call writes, and what it reads of others: whether any of the first meets anything else but its own source.
struct Range {
  Span span;
  int owner, source;  // source: what may lie under this output (an index of a matrix), or -1
  bool output;
  uintptr_t first() const { return reinterpret_cast<uintptr_t>(span.p); }
  uintptr_t end() const { return first() + (uintptr_t)((span.rows - 1) * span.ld + span.width); }
};
bool any_meet(std::vector<Range>& all) {
  all.erase(std::remove_if(all.begin(), all.end(), [](const Range& r) { return !r.span.p || r.span.rows <= 0 || r.span.width <= 0; }), all.end());
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.first() < b.first(); });
  std::vector<const Range*> open;
  for (const Range& r : all) {
    open.erase(std::remove_if(open.begin(), open.end(), [&](const Range* o) { return o->end() <= r.first(); }), open.end());
    for (const Range* o : open) {
      if (!r.output && !o->output) continue;
      const bool own = (r.output && !o->output && r.source == o->owner) || (o->output && !r.output && o->source == r.owner);
      if (!own && meet(r.span, o->span)) return true;
    }
    open.push_back(&r);
  }
  return false;
}

// What is small is a chain of launches, which company makes longer; what is nearly square gains little.  In us, one at a time / in company, bf16
// and fp32: 1024 x 256 107 / 113, 141 / 165; 8 of them 125 / 126, 174 / 176; 48 336 / 275, 465 / 375; 2048 x 512 131 / 138, 174 / 184; 12 of them 421 / 328,
// 669 / 478; 1280 x 1024 166 / 178, 308 / 300; 1536 x 1024 173 / 182, 351 / 317; 2048 x 1024 185 / 189, 329 / 309; 4096 x 1024 325 / 271, 509 / 383;
// 2400 x 2048 421 / 385, 824 / 852; 2560 x 2048 413 / 385, 833 / 852; 5120 x 4096 1806 / 1683, 4854 / 4802; 8192 x 2048 936 / 667, 1852 / 1294.  Near the
// thresholds, how many tiles are left for a last round decides more than they do, either way: 2600 x 2080 in bf16 561 / 653, 1700 x 1360 in fp32
// 479 / 413 are the most that the rule loses.
// In one term, what company leaves behind does not average out in small matrices: 33 of 145 x 2449, rank 20 to 60, 5.8e-3 off (one at a time 2e-3).
int steps_at_a_time(const MuonBatch& b) {
  if (b.terms == 1 && b.S < 256) return 1;
  const int64_t size = (int64_t)b.n * b.S * b.S, quarters = size < (1 << 22) ? 6 : 5;
  return size < (1 << 19) || 4 * (int64_t)b.L < quarters * b.S ? 1 : b.terms == 2 ? 3 : 2;
}

int run(const std::vector<Matrix>& all, const Plans& plans, const MuonBatch& common, void* workspace, cudaStream_t s) {
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != SFFN_OK) return rc;
  for (const auto& batch : batches_of(all)) {
    MuonBatch b = common;
    layout(b, (int)batch.size(), *batch[0], static_cast<char*>(workspace));
    for (size_t i = 0; i < batch.size(); ++i) b.item[i] = batch[i]->item;
    SFFN_CUDA(sffn::launch_muon_moments(b, sms, s));
    SFFN_CUDA(sffn::launch_muon_scale(b, sms, s));
    for (const sffn::MuonProduct& p : plans.of[steps_at_a_time(b) - 1]) SFFN_CUDA(sffn::launch_muon_product(b, p, sms, s));
  }
  return SFFN_OK;
}

// Terms of the products' operands.  Roundings of a matrix of a few singular values do not average out (2 x 6 up to 8e-3 off in one term), and two
// terms of so little cost no more than a tenth of the time.
int terms_of(int bits, bool wide, const Matrix& m) { return bits == 32 || (bits == 0 && wide) || std::min(m.R, m.C) < 8 ? 2 : 1; }

int matrices_of(const sffn_orthogonal* t, int n, const sffn_newton_schulz* ns, std::vector<Matrix>& out, bool pointers) {
  if (n < 0 || (n > 0 && !t)) return SFFN_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const sffn_orthogonal& a = t[i];
    if (!storage_type(a.dtype)) return SFFN_ERR_INVALID_ARG;
    const int shape = check_shape(a.rows, a.cols);
    if (shape != SFFN_OK) return shape;
    if (pointers && a.rows > 0 && a.cols > 0) {
      if (!a.u || !a.o || a.ld_u < a.cols || a.ld_o < a.cols) return SFFN_ERR_INVALID_ARG;
      if (!aligned(a.u, element(a.dtype)) || !aligned(a.o, element(a.dtype)) || a.ld_u > (1ll << 40) || a.ld_o > (1ll << 40)) return SFFN_ERR_UNSUPPORTED;
    }
    Matrix m{};
    m.item.src = a.u; m.item.ld_src = a.ld_u;
    m.item.out = a.o; m.item.ld_out = a.ld_o;
    m.R = a.rows; m.C = a.cols;
    m.src_bf16 = m.out_bf16 = a.dtype == SFFN_BF16;
    m.terms = terms_of(ns->bits, a.dtype == SFFN_F32, m);
    out.push_back(m);
  }
  return SFFN_OK;
}

int matrices_of(const sffn_muon_tensor* t, int n, const sffn_newton_schulz* ns, std::vector<Matrix>& out, bool pointers) {
  if (n < 0 || (n > 0 && !t)) return SFFN_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const sffn_muon_tensor& a = t[i];
    if (!storage_type(a.p_dtype) || !storage_type(a.g_dtype) || (a.master && a.p_dtype != SFFN_BF16)) return SFFN_ERR_INVALID_ARG;
    const int shape = check_shape(a.rows, a.cols);
    if (shape != SFFN_OK) return shape;
    if (pointers) {
      if (!std::isfinite(a.lr) || !std::isfinite(a.weight_decay) || !std::isfinite(a.scale)) return SFFN_ERR_INVALID_ARG;
      if (a.rows > 0 && a.cols > 0) {
        if (!a.p || !a.g || !a.m) return SFFN_ERR_INVALID_ARG;
        if (!aligned(a.p, element(a.p_dtype)) || !aligned(a.g, element(a.g_dtype)) || !aligned(a.m, 4) || !aligned(a.master, 4)) return SFFN_ERR_UNSUPPORTED;
      }
    }
    Matrix m{};
    m.item.src = a.g; m.item.ld_src = a.cols;
    m.item.out = a.p; m.item.ld_out = a.cols;
    m.item.m = a.m; m.item.master = a.master;
    m.item.decay = (float)(1.0 - a.lr * a.weight_decay);
    m.item.rate = (float)(a.lr * a.scale);
    m.R = a.rows; m.C = a.cols;
    m.src_bf16 = a.g_dtype == SFFN_BF16;
    m.out_bf16 = a.p_dtype == SFFN_BF16;
    m.terms = terms_of(ns->bits, a.p_dtype == SFFN_F32 || a.master, m);
    out.push_back(m);
  }
  return SFFN_OK;
}

template <typename T>
int workspace_bytes(const T* t, int n, const sffn_newton_schulz* ns, size_t* bytes) {
  if (!bytes) return SFFN_ERR_INVALID_ARG;
  const Plans* plans = nullptr;
  std::vector<Matrix> all;
  int rc = check_ns(ns, &plans);
  if (rc == SFFN_OK) rc = matrices_of(t, n, ns, all, false);
  if (rc == SFFN_OK) *bytes = workspace_of(all);
  return rc;
}

int check_workspace(const std::vector<Matrix>& all, const void* workspace, size_t bytes, const int32_t* status) {
  if (!status) return SFFN_ERR_INVALID_ARG;
  if (!aligned(status, 4)) return SFFN_ERR_UNSUPPORTED;
  return workspace && aligned(workspace, 256) && bytes >= workspace_of(all) ? SFFN_OK : SFFN_ERR_WORKSPACE;
}

// No exception leaves a C call: what the lists here need is little, but it is memory.
template <typename F>
int guarded(F f) {
  try {
    return f();
  } catch (...) {
    return SFFN_ERR_INVALID_ARG;
  }
}

}  // namespace

extern "C" {

int sffn_orthogonalize_workspace_bytes(const sffn_orthogonal* t, int n, const sffn_newton_schulz* ns, size_t* bytes) {
  return guarded([&] { return workspace_bytes(t, n, ns, bytes); });
}
int sffn_muon_workspace_bytes(const sffn_muon_tensor* t, int n, const sffn_newton_schulz* ns, size_t* bytes) {
  return guarded([&] { return workspace_bytes(t, n, ns, bytes); });
}

int sffn_orthogonalize(const sffn_orthogonal* t, int n, const sffn_newton_schulz* ns, void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  return guarded([&]() -> int {
    const Plans* plans = nullptr;
    std::vector<Matrix> all;
    int rc = check_ns(ns, &plans);
    if (rc == SFFN_OK) rc = matrices_of(t, n, ns, all, true);
    if (rc == SFFN_OK) rc = check_workspace(all, workspace, workspace_bytes, status);
    if (rc != SFFN_OK) return rc;
    std::vector<Range> ranges = {{whole(workspace, (int64_t)workspace_of(all)), -2, -1, true}, {whole(status, 4), -3, -1, true}};
    for (int i = 0; i < n; ++i) {
      const int64_t e = (int64_t)element(t[i].dtype), rows = t[i].rows, width = e * t[i].cols;
      ranges.push_back({{t[i].u, rows, width, e * t[i].ld_u}, i, -1, false});
      ranges.push_back({{t[i].o, rows, width, e * t[i].ld_o}, i, i, true});
    }
    if (any_meet(ranges)) return SFFN_ERR_INVALID_ARG;
    MuonBatch common{};
    common.eps = (float)ns->eps;
    common.status = status;
    return run(all, *plans, common, workspace, static_cast<cudaStream_t>(stream));
  });
}

int sffn_muon_step(const sffn_muon_tensor* t, int n, const sffn_muon_config* c, void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  return guarded([&]() -> int {
    if (!c) return SFFN_ERR_INVALID_ARG;
    const Plans* plans = nullptr;
    std::vector<Matrix> all;
    int rc = check_ns(&c->newton_schulz, &plans);
    if (rc != SFFN_OK) return rc;
    if (!(c->momentum >= 0 && c->momentum < 1) || (c->grad_norm && !(c->max_norm > 0))) return SFFN_ERR_INVALID_ARG;
    if (!aligned(c->grad_norm, 4)) return SFFN_ERR_UNSUPPORTED;
    rc = matrices_of(t, n, &c->newton_schulz, all, true);
    if (rc == SFFN_OK) rc = check_workspace(all, workspace, workspace_bytes, status);
    if (rc != SFFN_OK) return rc;
    std::vector<Range> ranges = {{whole(workspace, (int64_t)workspace_of(all)), -2, -1, true}, {whole(status, 4), -3, -1, true}, {whole(c->grad_norm, 4), -4, -1, false}};
    for (int i = 0; i < n; ++i) {
      const int64_t entries = (int64_t)t[i].rows * t[i].cols;
      ranges.push_back({whole(t[i].g, entries * (int64_t)element(t[i].g_dtype)), i, -1, false});
      ranges.push_back({whole(t[i].p, entries * (int64_t)element(t[i].p_dtype)), i, -1, true});
      ranges.push_back({whole(t[i].m, entries * 4), i, -1, true});
      ranges.push_back({whole(t[i].master, entries * 4), i, -1, true});
    }
    if (any_meet(ranges)) return SFFN_ERR_INVALID_ARG;
    MuonBatch common{};
    common.step = true;
    common.nesterov = c->nesterov != 0;
    common.momentum = (float)c->momentum;
    common.one_momentum = (float)(1.0 - c->momentum);
    common.eps = (float)c->newton_schulz.eps;
    common.grad_norm = c->grad_norm;
    common.max_norm = (float)c->max_norm;
    common.status = status;
    return run(all, *plans, common, workspace, static_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
