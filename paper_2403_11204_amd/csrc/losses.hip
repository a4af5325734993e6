// C ABI of the losses over the classes of a linear layer (see include/slp.h for the contract).  Host code only: every argument is checked
// before anything is queued.
#include "../../include/slp.h"

#include "class_loss.h"
#include "operator_checks.h"

using namespace slp;

namespace {

constexpr int kMaxRows = 1 << 20, kMaxDim = 1 << 20, kMaxTop = 1024;
// P of a piece of the classes takes this much at most, or what 256 classes take (the width of a tile), and the padding of its rows.
constexpr int64_t kPieceBytes = 256 << 20;
// Logits that are kept in float32 between the loss and the gradient, where they are wanted: what fits here without the padding of their rows.  A piece of others is computed twice, which takes the third of three products
// again.
constexpr int64_t kKeptBytes = (int64_t)1 << 30;
// A tile of 256 rows is addressed with 32-bit offsets: rows of x, W and P lie at most this many elements apart.
constexpr int kMaxPiece = 1 << 20;
constexpr int64_t kAcross = 0x7FFFFF00;
// Grids have fewer than 2^32 threads.
constexpr int64_t kMaxWeights = (int64_t)1 << 33, kMaxLogits = (int64_t)1 << 36, kMaxTargets = (int64_t)1 << 25;

// Rows of `width` elements on 128-byte boundaries, not a multiple of 4 KB apart where that many rows share few memory channels.
int64_t row_ld(int64_t width, int64_t es) {
  int64_t ld = (width * es + 127) / 128 * 128;
  if (ld % 4096 == 0) ld += 128;
  return ld / es;
}

struct Call {
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  const float* bias;
  Targets t;
  int dt, rows, classes, dim;
  float temperature, scale;
  float *loss, *losses, *lse;
  void* dx;
  int64_t lddx;
  void* dw;
  int64_t lddw;
  int dw_dt;
  float* dbias;
};

// Where everything lies in the workspace, and in which pieces the classes are taken.
struct Plan {
  int64_t es, ldk, ldp;                 // operands' element size; leading dimensions of copies of x and W, of P
  bool copy_x, copy_w, fix;
  int piece, kept;                      // classes of a piece; those whose logits are kept, whole pieces
  int64_t ldz;
  int dx_parts, dw_parts, z_parts, spans;
  size_t zt, p, labels, norm, alpha, means, stats, xc, wc, xz, z, z_work, P, dx_work, dw_work, sums, fixed, bytes;
};

// Whether the products can read a matrix in place.
bool in_place(const void* p, int64_t ld, int rows, int dim, int64_t es) { return !off(p, 16) && (rows == 1 || ld * es % 16 == 0) && dim * es % 16 == 0; }

// Classes from `first` on whose logits a launch takes: no more than the copy of W holds, and whole rounds of the chip where those are few.
int stats_columns(const Call& c, const Plan& a, int first) {
  const int left = a.copy_w ? a.piece - first % a.piece : c.classes, most = c.classes - first < left ? c.classes - first : left;
  return whole_rounds(c.dt, PRODUCT_STATS, most, c.rows, c.dim);
}

Plan plan_of(const Call& c) {
  Plan a{};
  const bool grads = c.dx || c.dw || c.dbias;
  a.es = (int64_t)size_of(c.dt);
  a.ldk = row_ld(c.dim, a.es);
  a.copy_x = !in_place(c.x, c.ldx, c.rows, c.dim, a.es);
  a.copy_w = !in_place(c.w, c.ldw, c.classes, c.dim, a.es);
  int64_t most = kPieceBytes / ((int64_t)c.rows * a.es) / 256 * 256;
  if (most < 256) most = 256;
  if (most > kMaxPiece) most = kMaxPiece;
  // W's piece and x are addressed with 32-bit offsets where they lie the other way (see class_loss.h)
  const int64_t across = kAcross / ((a.copy_w ? a.ldk : c.ldw) * a.es) / 256 * 256;
  if (c.classes > 1 && most > across) most = across;
  const int wanted = (int)((c.classes + most - 1) / most);
  a.piece = wanted == 1 ? c.classes : ((c.classes + wanted - 1) / wanted + 255) / 256 * 256;
  const int pieces = (c.classes + a.piece - 1) / a.piece;
  a.ldp = row_ld(a.piece, a.es);
  if (pieces == 1) a.z_parts = z_parts(c.dt, c.rows, c.classes, c.dim);
  if (grads || a.z_parts) {
    const int64_t fit = kKeptBytes / ((int64_t)c.rows * 4);
    a.kept = fit >= c.classes ? c.classes : (int)(fit / a.piece) * a.piece;
    a.ldz = row_ld(a.kept, 4);
  }
  a.dx_parts = class_parts(c.dt, c.rows, c.dim, a.piece);
  a.dw_parts = class_parts(c.dt, a.piece, c.dim, c.rows);
  for (int first = 0, columns; first < c.classes; first += columns) {
    columns = stats_columns(c, a, first);
    a.spans += stats_spans(c.dt, c.rows, columns, c.dim);
  }
  size_t at = 0;
  auto take = [&](bool wanted, int64_t bytes) {
    const size_t here = at;
    if (wanted) at += ((size_t)bytes + 255) & ~(size_t)255;
    return here;
  };
  const int64_t targets = (int64_t)c.rows * c.t.k, r = c.rows, dq = (c.dim + 3) / 4 * 4;
  a.zt = take(true, targets * 4);
  a.p = take(c.t.top, targets * 4);
  a.labels = take(!c.t.top, r * 4);
  a.norm = take(true, r * 8);
  a.alpha = take(true, 4);
  a.means = take(true, r * 16);
  a.stats = take(a.z_parts == 0, (int64_t)a.spans * r * 8);
  a.xc = take(a.copy_x, r * a.ldk * a.es);
  a.wc = take(a.copy_w, (int64_t)a.piece * a.ldk * a.es);
  a.xz = a.copy_x ? a.xc : take(c.dw, r * a.ldk * a.es);
  a.z = take(a.kept > 0, r * a.ldz * 4);
  a.z_work = take(a.z_parts > 0, a.z_parts * r * ((c.classes + 3) / 4 * 4) * 4);
  a.P = take(grads, r * a.ldp * a.es);
  a.dx_work = take(c.dx && (pieces > 1 || a.dx_parts > 1), (int64_t)a.dx_parts * r * dq * 4);
  a.dw_work = take(c.dw && a.dw_parts > 1, (int64_t)a.dw_parts * a.piece * dq * 4);
  // sums of a piece's columns, over as many parts of the rows as the widest kernel makes
  const int64_t rest = c.classes - (int64_t)(pieces - 1) * a.piece, most_sums = (int64_t)sum_parts(c.dt, c.rows, a.piece, c.dim) * a.piece;
  const int64_t rest_sums = rest > 0 ? sum_parts(c.dt, c.rows, (int)rest, c.dim) * rest : 0;      // (smaller tiles, more parts)
  const int64_t kept_piece = (int64_t)kept_sum_parts(c.rows, a.piece) * a.piece, kept_rest = rest > 0 ? kept_sum_parts(c.rows, (int)rest) * rest : 0;
  const int64_t kept_sums = kept_piece > kept_rest ? kept_piece : kept_rest, gemm_sums = most_sums > rest_sums ? most_sums : rest_sums;
  a.sums = take(c.dbias, (kept_sums > gemm_sums ? kept_sums : gemm_sums) * 4);
  // a distillation's targets among pieces that do not see to them while they are turned into P
  a.fix = c.dbias && c.t.top && (a.kept < c.classes || !fixes_targets(c.t.k, a.piece));
  a.fixed = take(a.fix, (int64_t)c.classes * 8);
  a.bytes = at;
  return a;
}

int run(const Call& c, void* workspace, hipStream_t s) {
  const Plan a = plan_of(c);
  char* const base = (char*)workspace;
  auto at = [&](size_t offset) { return base + offset; };
  float *const zt = (float*)at(a.zt), *const p = (float*)at(a.p), *const alpha = (float*)at(a.alpha);
  float2* const norm = (float2*)at(a.norm);
  const float per_t = 1.0f / c.temperature;
  const bool grads = c.dx || c.dw || c.dbias;

  const void* x = c.x;
  int64_t ldx = c.rows == 1 ? a.ldk : c.ldx;       // (a single row may have any)
  if (a.copy_x) {
    HIP_TRY(launch_pad_rows(c.dt, c.x, c.ldx, c.rows, c.dim, at(a.xc), a.ldk, s));
    x = at(a.xc);
    ldx = a.ldk;
  }
  // W's rows from class `first` on, where the products can read them
  int copied = -1;                       // what the copy holds
  auto weights = [&](int first, int columns, const void*& w, int64_t& ldw) -> int {
    w = (const char*)c.w + (int64_t)first * c.ldw * a.es;
    ldw = c.classes == 1 ? a.ldk : c.ldw;
    if (a.copy_w) {
      if (copied != first) HIP_TRY(launch_pad_rows(c.dt, w, c.ldw, columns, c.dim, at(a.wc), a.ldk, s));
      copied = first;
      w = at(a.wc);
      ldw = a.ldk;
    }
    return SLP_OK;
  };
  if (a.kept < c.classes) HIP_TRY(launch_target_logits(c.dt, TargetLogits{c.x, c.w, c.ldx, c.ldw, c.bias, c.rows, c.classes, c.dim, a.kept, c.t, zt}, s));
  float* const z = a.kept ? (float*)at(a.z) : nullptr;
  float2* stats = (float2*)at(a.stats);
  for (int first = 0, columns; first < c.classes; first += columns) {
    columns = a.z_parts ? c.classes : stats_columns(c, a, first);
    ClassProduct g{};
    const int from = a.copy_w ? first % a.piece : 0, held = c.classes - (first - from) < a.piece ? c.classes - (first - from) : a.piece;
    SLP_CHECK(weights(first - from, held, g.b, g.ldb));
    g.b = (const char*)g.b + (a.copy_w ? (int64_t)from * g.ldb * a.es : 0);
    g.a = x;
    g.lda = ldx;
    g.M = c.rows;
    g.N = columns;
    g.K = c.dim;
    g.bias = c.bias ? c.bias + first : nullptr;
    g.per_t = per_t;
    g.stats = stats;
    if (first < a.kept) {
      g.z = z + first;
      g.ldz = a.ldz;
      g.zcols = a.kept - first < columns ? a.kept - first : columns;
    }
    g.parts = 1;
    if (a.z_parts) {                     // (one piece: all classes)
      g.work = (float*)at(a.z_work);
      g.parts = a.z_parts;
    }
    HIP_TRY(launch_class_product(c.dt, a.z_parts ? PRODUCT_Z : PRODUCT_STATS, g, s));
    stats += (int64_t)stats_spans(c.dt, c.rows, columns, c.dim) * c.rows;
  }
  unsigned long long* const all_fixed = a.fix ? (unsigned long long*)at(a.fixed) : nullptr;
  int32_t* const labels = c.t.top ? nullptr : (int32_t*)at(a.labels);
  RowLoss each{(const float2*)at(a.stats), a.spans, a.z_parts ? (const float*)at(a.z_work) : nullptr, a.z_parts, c.bias, c.rows, c.classes, c.t, z, a.ldz, a.kept, zt, c.temperature * c.temperature, c.lse, c.losses, norm, p, labels, all_fixed, (double2*)at(a.means), nullptr};
  const bool alone = !grads && row_groups(each) == 1;
  if (alone) each.loss = c.loss;
  HIP_TRY(launch_row_loss(each, s));
  // (xz: the rows that count; 0 times what others hold may be NaN)
  const AllRows all{each.means, row_groups(each), norm, c.rows, c.dim, c.scale * c.temperature, c.loss, alpha, a.copy_x ? nullptr : c.x, c.ldx, c.dw ? at(a.xz) : nullptr, a.ldk};
  if ((!a.kept || !grads) && !alone) HIP_TRY(launch_all_rows(c.dt, all, s));
  if (!grads) return SLP_OK;

  for (int first = 0; first < c.classes; first += a.piece) {
    const int columns = c.classes - first < a.piece ? c.classes - first : a.piece;
    const bool last = first + columns == c.classes;
    const bool kept = first < a.kept;
    const void* w = nullptr;
    int64_t ldw = 0;
    if (!kept || c.dx) SLP_CHECK(weights(first, columns, w, ldw));
    float* const sums = c.dbias ? (float*)at(a.sums) : nullptr;
    unsigned long long* const fixed = all_fixed ? all_fixed + first : nullptr;
    const TargetFix fix{c.t, c.rows, c.classes, c.dt, zt, p, norm, first, columns, at(a.P), a.ldp, fixed, sums};
    if (kept) {
      HIP_TRY(launch_kept_prob(fix, z + first, a.ldz, labels, first == 0 ? &all : nullptr, s));
    } else {
      ClassProduct g{};
      g.a = x;
      g.lda = ldx;
      g.b = w;
      g.ldb = ldw;
      g.M = c.rows;
      g.N = columns;
      g.K = c.dim;
      g.bias = c.bias ? c.bias + first : nullptr;
      g.per_t = per_t;
      g.norm = norm;
      g.labels = labels;
      g.label0 = first;
      g.p = at(a.P);
      g.ldp = a.ldp;
      g.sums = sums;
      g.parts = 1;
      HIP_TRY(launch_class_product(c.dt, PRODUCT_PROB, g, s));
      if (c.t.top) HIP_TRY(launch_target_fix(fix, s));
    }
    const BiasGradient bias{sums, kept ? kept_sum_parts(c.rows, columns) : sum_parts(c.dt, c.rows, columns, c.dim), columns, fixed, alpha, c.dbias + first};
    bool bias_left = c.dbias;              // (goes along with the first joining of parts)
    auto join = [&](int dt, const float* work, int parts, int rows, void* out, int64_t ldo) -> int {
      HIP_TRY(launch_join_parts(dt, work, parts, rows, c.dim, alpha, out, ldo, bias_left ? &bias : nullptr, s));
      bias_left = false;
      return SLP_OK;
    };
    ClassProduct dx{}, dw{};
    if (c.dx) {
      dx.a = at(a.P);
      dx.lda = a.ldp;
      dx.b = w;
      dx.ldb = ldw;
      dx.M = c.rows;
      dx.N = c.dim;
      dx.K = columns;
      dx.alpha = alpha;
      dx.parts = a.dx_parts;
      if (a.dx_parts > 1 || a.piece < c.classes) {
        dx.work = (float*)at(a.dx_work);
        dx.add = first > 0;
      } else {
        dx.out = c.dx;
        dx.ldo = c.lddx;
        dx.out_dtype = c.dt;
      }
    }
    if (c.dw) {
      dw.a = at(a.P);
      dw.lda = a.ldp;
      dw.b = at(a.xz);
      dw.ldb = a.ldk;
      dw.M = columns;
      dw.N = c.dim;
      dw.K = c.rows;
      dw.alpha = alpha;
      dw.parts = a.dw_parts;
      if (a.dw_parts > 1) {
        dw.work = (float*)at(a.dw_work);
      } else {
        dw.out = (char*)c.dw + (int64_t)first * c.lddw * (int64_t)size_of(c.dw_dt);
        dw.ldo = c.lddw;
        dw.out_dtype = c.dw_dt;
      }
    }
    bool together = false;
    if (c.dx && c.dw) HIP_TRY(launch_class_gradients(c.dt, dx, dw, together, s));
    else if (c.dx) HIP_TRY(launch_class_product(c.dt, PRODUCT_DX, dx, s));
    if (dx.work && last) SLP_CHECK(join(c.dt, dx.work, dx.parts, c.rows, c.dx, c.lddx));
    if (c.dw) {
      const int most = dw.work ? columns : whole_rounds(c.dt, PRODUCT_DW, columns, c.dim, c.rows);
      if (!together) {
        dw.M = most;
        HIP_TRY(launch_class_product(c.dt, PRODUCT_DW, dw, s));
        if (most < columns) {
          dw.a = (const char*)dw.a + most * a.es;
          dw.out = (char*)dw.out + (int64_t)most * c.lddw * (int64_t)size_of(c.dw_dt);
          dw.M = columns - most;
          HIP_TRY(launch_class_product(c.dt, PRODUCT_DW, dw, s));
        }
      }
      if (dw.work) SLP_CHECK(join(c.dw_dt, dw.work, dw.parts, columns, (char*)c.dw + (int64_t)first * c.lddw * (int64_t)size_of(c.dw_dt), c.lddw));
    }
    if (bias_left) SLP_CHECK(join(c.dt, nullptr, 0, 0, nullptr, 0));
  }
  return SLP_OK;
}

// Sizes and leading dimensions that plan_of takes: it divides by them.
int check_sizes(const char* who, const Call& c) {
  if (c.rows < 0 || c.classes <= 0 || c.dim <= 0) return fail(SLP_ERR_ARG, "%s: rows %d, classes %d, dim %d", who, c.rows, c.classes, c.dim);
  if (c.rows > kMaxRows || c.classes > kMaxSide || c.dim > kMaxDim)
    return fail(SLP_ERR_SHAPE, "%s: up to %d rows, %d classes and a width of %d (got %d, %d, %d)", who, kMaxRows, kMaxSide, kMaxDim, c.rows, c.classes, c.dim);
  if ((int64_t)c.classes * c.dim > kMaxWeights || (int64_t)c.rows * c.dim > kMaxWeights || (int64_t)c.rows * c.classes > kMaxLogits || (int64_t)c.rows * c.t.k > kMaxTargets)
    return fail(SLP_ERR_SHAPE, "%s: %d rows of %d and %d classes, %d targets a row", who, c.rows, c.dim, c.classes, c.t.k);
  return SLP_OK;
}
int check_rows(const char* who, const Call& c) {
  SLP_CHECK(check_dense(who, "x", c.x, c.ldx, c.dim, c.dt));
  SLP_CHECK(check_dense(who, "w", c.w, c.ldw, c.dim, c.dt));
  if (c.dw && c.rows * row_ld(c.dim, (int64_t)size_of(c.dt)) * (int64_t)size_of(c.dt) >= kAcross) return fail(SLP_ERR_SHAPE, "%s: %d rows of %d come to 2 GiB", who, c.rows, c.dim);
  if ((c.rows > 1 && c.ldx > kMaxPiece) || (c.classes > 1 && c.ldw > kMaxPiece)) return fail(SLP_ERR_SHAPE, "%s: rows of x and w lie at most %d elements apart", who, kMaxPiece);
  return SLP_OK;
}

int check_call(const char* who, const Call& c) {
  if (!known(c.dt) || (c.dw && !known(c.dw_dt))) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, known(c.dt) ? c.dw_dt : c.dt);
  SLP_CHECK(check_sizes(who, c));
  if (!(c.scale == c.scale) || c.scale - c.scale != 0.0f) return fail(SLP_ERR_ARG, "%s: the gradients' scale must be finite", who);
  if (!c.loss) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  if (off(c.loss, 4) || off(c.losses, 4) || off(c.lse, 4) || off(c.bias, 4) || off(c.dbias, 4))
    return fail(SLP_ERR_ALLOC, "%s: a float32 vector is not on an element's boundary", who);
  if (c.dw) SLP_CHECK(check_dense(who, "dw", c.dw, c.lddw, c.dim, c.dw_dt));
  if (c.rows == 0) return SLP_OK;
  if (!c.x || !c.w || !c.t.ids || !c.losses || !c.lse) return fail(SLP_ERR_ARG, "%s: null pointer", who);
  SLP_CHECK(check_rows(who, c));
  if (c.dx) SLP_CHECK(check_dense(who, "dx", c.dx, c.lddx, c.dim, c.dt));
  if (off(c.t.ids, c.t.ids64 ? 8 : 4)) return fail(SLP_ERR_ALLOC, "%s: class ids are not on an element's boundary", who);
  return SLP_OK;
}

// What no rows leave: a loss of zero, gradients of zero.
int nothing(const Call& c, hipStream_t s) {
  HIP_TRY(launch_zero(SLP_F32, c.loss, 1, 1, 1, s));
  if (c.dbias) HIP_TRY(launch_zero(SLP_F32, c.dbias, c.classes, 1, c.classes, s));
  if (c.dw) HIP_TRY(launch_zero(c.dw_dt, c.dw, c.lddw, c.classes, c.dim, s));
  return SLP_OK;
}

int loss_call(const char* who, const Call& c, void* workspace, size_t workspace_bytes, hipStream_t s) {
  if (c.rows == 0) return nothing(c, s);
  SLP_CHECK(check_work(who, workspace, workspace_bytes, plan_of(c).bytes));
  return run(c, workspace, s);
}

}  // namespace

extern "C" {

size_t slp_linear_loss_workspace_bytes(const void* x, int64_t ldx, const void* w, int64_t ldw, int dt, int rows, int classes, int dim, int top, int outputs) {
  const char* const who = "slp_linear_loss_workspace_bytes";
  if (!known(dt) || rows <= 0 || top < 0 || top > kMaxTop) return 0;
  static char given;
  Call c{};
  c.x = x;
  c.ldx = ldx;
  c.w = w;
  c.ldw = ldw;
  c.dt = dt;
  c.rows = rows;
  c.classes = classes;
  c.dim = dim;
  c.t.k = top ? top : 1;
  c.t.top = top ? &given : nullptr;
  c.dx = outputs & SLP_LOSS_DX ? &given : nullptr;
  c.dw = outputs & SLP_LOSS_DW ? &given : nullptr;
  c.dbias = outputs & SLP_LOSS_DBIAS ? (float*)&given : nullptr;
  // (the binding asks for the workspace before the call that reports what is out of range)
  return check_sizes(who, c) || check_rows(who, c) ? 0 : plan_of(c).bytes;
}

int slp_linear_cross_entropy(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, int dt, int rows, int classes, int dim, const void* targets,
                             int target_bytes, float scale, float* loss, float* losses, float* lse, void* dx, int64_t lddx, void* dw, int64_t lddw, int dw_dt,
                             float* dbias, void* workspace, size_t workspace_bytes, slp_stream stream) {
  const char* const who = "slp_linear_cross_entropy";
  if (target_bytes != 4 && target_bytes != 8) return fail(SLP_ERR_ARG, "%s: class ids of 4 or 8 bytes (got %d)", who, target_bytes);
  const Targets t{targets, 1, target_bytes == 8, nullptr, 0, 0, 1, 1.0f};
  const Call c{x, ldx, w, ldw, bias, t, dt, rows, classes, dim, 1.0f, scale, loss, losses, lse, dx, lddx, dw, lddw, dw_dt, dbias};
  SLP_CHECK(check_call(who, c));
  return loss_call(who, c, workspace, workspace_bytes, (hipStream_t)stream);
}

int slp_linear_distillation(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias, int dt, int rows, int classes, int dim, const void* top, int64_t ldtop,
                            int top_dt, const void* top_classes, int64_t ldclasses, int class_bytes, int k, float temperature, float scale, float* loss, float* losses,
                            float* lse, void* dx, int64_t lddx, void* dw, int64_t lddw, int dw_dt, float* dbias, void* workspace, size_t workspace_bytes,
                            slp_stream stream) {
  const char* const who = "slp_linear_distillation";
  if (class_bytes != 4 && class_bytes != 8) return fail(SLP_ERR_ARG, "%s: class ids of 4 or 8 bytes (got %d)", who, class_bytes);
  if (!known(top_dt)) return fail(SLP_ERR_ARG, "%s: unknown dtype %d", who, top_dt);
  if (k <= 0 || k > kMaxTop) return fail(SLP_ERR_ARG, "%s: 1 to %d of the teacher's logits a row (got %d)", who, kMaxTop, k);
  if (!(temperature >= 1e-3f && temperature <= 1e3f)) return fail(SLP_ERR_ARG, "%s: a temperature between 0.001 and 1000 (got %g)", who, (double)temperature);
  const Targets t{top_classes, ldclasses, class_bytes == 8, top, ldtop, top_dt, k, 1.0f / temperature};
  const Call c{x, ldx, w, ldw, bias, t, dt, rows, classes, dim, temperature, scale, loss, losses, lse, dx, lddx, dw, lddw, dw_dt, dbias};
  SLP_CHECK(check_call(who, c));
  if (rows > 0) {
    if (!top) return fail(SLP_ERR_ARG, "%s: null pointer", who);
    SLP_CHECK(check_dense(who, "top", top, ldtop, k, top_dt));
    if (ldclasses < k || ldclasses > kMaxLd) return fail(SLP_ERR_SHAPE, "%s: leading dimension %lld of the classes, rows of %d", who, (long long)ldclasses, k);
  }
  return loss_call(who, c, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
