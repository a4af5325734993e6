// The operators' way from Python tensors to the C ABI (include/slp.h): argument checks, room for the outputs and workspaces from torch's
// allocator, the call.  An operator on a few rows takes the device 3 to 5 us; written in Python these steps took the host 10 to 17 us
// a call, here 5 with one launch, 8 to 12 with two.  Each function returns its outputs, or the library's error code as an integer.  A call runs on the device
// that its tensors are on, whichever is current, and on torch's current stream of that device.
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <string>
#include <vector>

#include "../../include/slp.h"

namespace {

// A failed check of an argument: AssertionError in Python.
struct Refused {
  std::string what;
};
void require(bool ok, const char* what) {
  if (!ok) throw Refused{what};
}

const at::Tensor& tensor(PyObject* o) {
  require(THPVariable_Check(o), "a tensor is wanted");
  return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }
int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}
// Sizes beyond int are refused by the library, as -1 is.
int side(int64_t n) { return n <= INT32_MAX ? (int)n : -1; }

int dtype_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return SLP_BF16;
  require(t.scalar_type() == at::kFloat, "float32 or bfloat16 is wanted");
  return SLP_F32;
}

// Leading dimension of a matrix on the device whose rows are contiguous; a side of one element may have any stride.
int64_t leading(const at::Tensor& t) {
  require(t.is_cuda() && t.dim() == 2, "a matrix on the device is wanted");
  const int64_t m = t.size(0), n = t.size(1), ld = t.stride(0);
  require(t.stride(1) == 1 || n <= 1, "rows must be contiguous");
  return m <= 1 && ld < n ? n : ld;
}
// The same of one of x's shape, type and place.
int64_t like(const at::Tensor& t, const at::Tensor& x) {
  require(t.scalar_type() == x.scalar_type() && t.sizes() == x.sizes() && t.device() == x.device(), "matrices of one shape, type and device are wanted");
  return leading(t);
}
// A contiguous float32 vector of n elements beside x, or null for None.
const float* vector(PyObject* o, int64_t n, const at::Tensor& x) {
  if (!given(o)) return nullptr;
  const at::Tensor& t = tensor(o);
  require(t.device() == x.device() && t.scalar_type() == at::kFloat && t.is_contiguous() && t.numel() == n, "a contiguous float32 vector on the same device is wanted");
  return (const float*)t.data_ptr();
}

// The tensors' device, current as long as this lives, and torch's current stream of it.  (A guard, and what a stream asks to find its handle, take the host
// half a microsecond each: not where the device is the current one already, the stream the default one, whose handle is null.)
class On {
 public:
  explicit On(const at::Device& device) {
    if (c10::hip::current_device() != device.index()) guard_.reset_device(device);
    const c10::hip::HIPStream s = c10::hip::getCurrentHIPStream(device.index());
    stream_ = s == c10::hip::getDefaultHIPStream(device.index()) ? nullptr : s.stream();
  }
  slp_stream stream() const { return stream_; }

 private:
  c10::OptionalDeviceGuard guard_;
  slp_stream stream_ = nullptr;
};

// Room for a call's outputs and workspace.  Each allocation takes the host 0.6 us: where all of them come to 256 KB at most (a request's
// rows: the device is done before the host) they are parts of one, on 256-byte boundaries.  A workspace only up to 4 KB: whatever output is kept keeps the block.
class Room {
 public:
  Room(const at::Device& device, size_t outputs, size_t workspace) : device_(device), apart_(workspace > 4096) {
    const size_t all = outputs + (apart_ ? 0 : padded(workspace));
    if (all <= (256u << 10)) block_ = at::empty({(int64_t)all}, at::TensorOptions().dtype(at::kByte).device(device));
  }
  static size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
  at::Tensor take(at::IntArrayRef sizes, at::ScalarType type) {
    if (!block_.defined()) return at::empty(sizes, at::TensorOptions().dtype(type).device(device_));
    at::Tensor t = at::detail::make_tensor<at::TensorImpl>(c10::Storage(block_.storage()), block_.key_set(), c10::scalarTypeToTypeMeta(type));
    const size_t size = t.itemsize();
    t.unsafeGetTensorImpl()->set_storage_offset((int64_t)(used_ / size));
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    used_ += padded((size_t)t.numel() * size);
    require(used_ <= block_.nbytes(), "room counted too small");
    return t;
  }
  at::Tensor work(size_t n) {
    if (!n) return at::Tensor();
    return apart_ ? at::empty({(int64_t)n}, at::TensorOptions().dtype(at::kByte).device(device_)) : take({(int64_t)n}, at::kByte);
  }

 private:
  at::Device device_;
  bool apart_;
  at::Tensor block_;
  size_t used_ = 0;
};
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// A matrix in 8 bits.
struct Eight {
  at::Tensor q, scales;
  void *at = nullptr, *scales_at = nullptr;
  int64_t ld = 0, lds = 0;
};
// Room for one: rows on 128-byte boundaries and, where there are many, not a multiple of 4 KB apart; rows of scales on 4-byte boundaries.
int64_t eight_ld(int64_t rows, int64_t cols) {
  const int64_t ld = (cols + 127) / 128 * 128;
  return ld % 4096 == 0 && rows > 16 ? ld + 128 : ld;
}
int64_t eight_lds(int64_t cols) { return (cols + 511) / 512 * 4; }
size_t eight_bytes(int64_t rows, int64_t cols, int64_t block) {
  return Room::padded((size_t)(rows * eight_ld(rows, cols))) + Room::padded((size_t)((rows + block - 1) / block * eight_lds(cols)));
}
Eight eight_room(int64_t rows, int64_t cols, int64_t block, Room& room) {
  Eight e;
  const int64_t blocks = (cols + 127) / 128, srows = (rows + block - 1) / block;
  e.ld = eight_ld(rows, cols);
  e.lds = eight_lds(cols);
  e.q = room.take({rows, e.ld}, at::kFloat8_e4m3fn);
  e.scales = room.take({srows, e.lds}, at::kFloat8_e8m0fnu);
  e.at = e.q.data_ptr();
  e.scales_at = e.scales.data_ptr();
  // (in place: each as_strided takes the host another half microsecond)
  if (e.ld != cols) e.q.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef({rows, cols}), at::IntArrayRef({e.ld, 1}));
  if (e.lds != blocks) e.scales.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef({srows, blocks}), at::IntArrayRef({e.lds, 1}));
  return e;
}
Eight eight_given(PyObject* q, PyObject* scales, int64_t block, int64_t cols) {
  Eight e;
  e.q = tensor(q);
  e.scales = tensor(scales);
  require(block == 1 || block == 128, "blocks of 1 or 128 rows");
  require(e.q.is_cuda() && e.q.dim() == 2 && e.q.scalar_type() == at::kFloat8_e4m3fn && e.q.size(1) == cols, "values of float8_e4m3fn with as many columns are wanted");
  require(e.scales.device() == e.q.device() && e.scales.dim() == 2 && e.scales.scalar_type() == at::kFloat8_e8m0fnu && e.scales.size(0) == (e.q.size(0) + block - 1) / block &&
              e.scales.size(1) == (cols + 127) / 128,
          "scales of float8_e8m0fnu, one for each block, are wanted");
  require((e.q.stride(1) == 1 || cols <= 1) && (e.scales.stride(1) == 1 || cols <= 128), "rows must be contiguous");
  e.at = e.q.data_ptr();
  e.scales_at = e.scales.data_ptr();
  // (a single row may have any stride; what it is read with beyond its end lies in the same 16 or 4 bytes)
  e.ld = e.q.size(0) <= 1 ? (cols + 15) / 16 * 16 : e.q.stride(0);
  e.lds = e.scales.size(0) <= 1 ? ((cols + 127) / 128 + 3) / 4 * 4 : e.scales.stride(0);
  return e;
}

PyObject* wrapped(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<at::Tensor> outputs) {
  THPObjectPtr all(PyTuple_New((Py_ssize_t)outputs.size()));
  if (!all) throw python_error();
  Py_ssize_t i = 0;
  for (const at::Tensor& t : outputs) {
    PyObject* o = wrapped(t);
    if (!o) throw python_error();
    PyTuple_SET_ITEM(all.get(), i++, o);
  }
  return all.release();
}
PyObject* code(int c) { return PyLong_FromLong(c); }

// x, block, rows, transposed, mask, column_sums
PyObject* quantize(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const int64_t block = integer(a[1]), ldx = leading(x), m = x.size(0), n = x.size(1);
  const int dt = dtype_of(x);
  require(block == 1 || block == 128, "blocks of 1 or 128 rows");
  int64_t ldmask = 0;
  const void* mask = nullptr;
  if (given(a[4])) {
    ldmask = like(tensor(a[4]), x);
    mask = tensor(a[4]).data_ptr();
  }
  const bool rows = truth(a[2]), transposed = truth(a[3]), column_sums = truth(a[5]);
  const size_t size = column_sums ? slp_quantize_workspace_bytes(side(m), side(n)) : 0;
  const On on(x.device());
  Room room(x.device(), (rows ? eight_bytes(m, n, block) : 0) + (transposed ? eight_bytes(n, m, block) : 0) + (column_sums ? Room::padded(4 * n) : 0), size);
  Eight r, t;
  if (rows) r = eight_room(m, n, block, room);
  if (transposed) t = eight_room(n, m, block, room);
  at::Tensor sums;
  if (column_sums) sums = room.take({n}, at::kFloat);
  const at::Tensor work = room.work(size);
  const int rc = slp_quantize(x.data_ptr(), ldx, mask, ldmask, dt, side(m), side(n), (int)block, r.at, r.ld, r.scales_at, r.lds, t.at, t.ld, t.scales_at, t.lds,
                              (float*)address(sums), address(work), size, on.stream());
  return rc ? code(rc) : tuple({r.q, r.scales, t.q, t.scales, sums});
}

// a's values, scales, block, b's, bias, relu, dtype, out, float32_sums
PyObject* product(PyObject* const* a) {
  const int64_t cols = tensor(a[0]).size(-1);
  const int64_t ablock = integer(a[2]), bblock = integer(a[5]);
  const Eight x = eight_given(a[0], a[1], ablock, cols), y = eight_given(a[3], a[4], bblock, cols);
  const int64_t m = x.q.size(0), n = y.q.size(0);
  require(x.q.device() == y.q.device(), "matrices on one device are wanted");
  const size_t size = slp_product_workspace_bytes(side(m), side(n), side(cols));
  at::Tensor out;
  int dt = (int)integer(a[8]);
  int64_t ldo = n;
  const On on(x.q.device());
  Room room(x.q.device(), given(a[9]) ? 0 : Room::padded((size_t)(m * n) * (dt == SLP_BF16 ? 2 : 4)), size);
  if (given(a[9])) {
    out = tensor(a[9]);
    require(out.dim() == 2 && out.size(0) == m && out.size(1) == n && out.device() == x.q.device(), "an output of the product's shape is wanted");
    ldo = leading(out);
    dt = dtype_of(out);
  } else {
    out = room.take({m, n}, dt == SLP_BF16 ? at::kBFloat16 : at::kFloat);
  }
  const at::Tensor work = room.work(size);
  const int rc = slp_product(x.at, x.ld, x.scales_at, x.lds, (int)ablock, y.at, y.ld, y.scales_at, y.lds, (int)bblock, vector(a[6], n, x.q), truth(a[7]), side(m), side(n),
                             side(cols), out.data_ptr(), ldo, truth(a[10]) ? dt | SLP_FLOAT32_SUMS : dt, address(work), size, on.stream());
  if (rc) return code(rc);
  return wrapped(out);
}

// A matrix of integers: its leading dimension and scales.
const float* integers_given(PyObject* q, PyObject* scales, int64_t cols, int64_t& ld) {
  const at::Tensor& t = tensor(q);
  require(t.is_cuda() && t.dim() == 2 && t.scalar_type() == at::kChar && t.size(1) == cols, "values of int8 with as many columns are wanted");
  require(t.stride(1) == 1 || cols <= 1, "rows must be contiguous");
  ld = t.size(0) <= 1 ? (cols + 15) / 16 * 16 : t.stride(0);
  require(given(scales), "scales of float32, one a row, are wanted");
  return vector(scales, t.size(0), t);
}

// x, out's values, scales
PyObject* quantize_integers(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const int64_t ldx = leading(x), m = x.size(0), n = x.size(1), end = (n + 15) / 16 * 16;
  const int dt = dtype_of(x);
  const On on(x.device());
  int64_t ld = eight_ld(m, n);
  at::Tensor q, scales;
  if (given(a[1])) {
    integers_given(a[1], a[2], n, ld);
    q = tensor(a[1]);
    scales = tensor(a[2]);
    require(q.size(0) == m && q.device() == x.device(), "an output of the matrix's shape is wanted");
    // (rows are written up to the next multiple of 16)
    require(m == 0 || n == 0 || q.storage_offset() + (m - 1) * ld + end <= (int64_t)q.storage().nbytes(), "an output whose rows have room for whole 16 bytes is wanted");
  } else {
    Room room(x.device(), Room::padded((size_t)(m * ld)) + Room::padded(4 * m), 0);
    q = room.take({m, ld}, at::kChar);
    scales = room.take({m}, at::kFloat);
    if (ld != n) q.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef({m, n}), at::IntArrayRef({ld, 1}));
  }
  const int rc = slp_quantize_integers(x.data_ptr(), ldx, dt, side(m), side(n), q.data_ptr(), ld, (float*)scales.data_ptr(), on.stream());
  return rc ? code(rc) : tuple({q, scales});
}

// a's values, scales, b's, bias, relu, dtype, out
PyObject* product_integers(PyObject* const* a) {
  const at::Tensor &x = tensor(a[0]), &y = tensor(a[2]);
  const int64_t cols = x.size(-1);
  int64_t lda, ldb;
  const float *const sa = integers_given(a[0], a[1], cols, lda), *const sb = integers_given(a[2], a[3], cols, ldb);
  require(x.device() == y.device(), "matrices on one device are wanted");
  const int64_t m = x.size(0), n = y.size(0);
  const size_t size = slp_product_integers_workspace_bytes(side(m), side(n), side(cols));
  at::Tensor out;
  int dt = (int)integer(a[6]);
  int64_t ldo = n;
  const On on(x.device());
  Room room(x.device(), given(a[7]) ? 0 : Room::padded((size_t)(m * n) * (dt == SLP_BF16 ? 2 : 4)), size);
  if (given(a[7])) {
    out = tensor(a[7]);
    require(out.dim() == 2 && out.size(0) == m && out.size(1) == n && out.device() == x.device(), "an output of the product's shape is wanted");
    ldo = leading(out);
    dt = dtype_of(out);
  } else {
    out = room.take({m, n}, dt == SLP_BF16 ? at::kBFloat16 : at::kFloat);
  }
  const at::Tensor work = room.work(size);
  const int rc = slp_product_integers(x.data_ptr(), lda, sa, y.data_ptr(), ldb, sb, vector(a[4], n, x), truth(a[5]), side(m), side(n), side(cols), out.data_ptr(), ldo, dt,
                                      address(work), size, on.stream());
  if (rc) return code(rc);
  return wrapped(out);
}

// x, gamma, residual, eps, normed, quantized
PyObject* rmsnorm(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const int64_t ldx = leading(x), m = x.size(0), n = x.size(1);
  const int dt = dtype_of(x);
  const float* gamma = vector(a[1], n, x);
  const bool normed = truth(a[4]), quantized = truth(a[5]);
  const size_t matrix = Room::padded((size_t)(m * n) * (dt == SLP_BF16 ? 2 : 4));
  const On on(x.device());
  Room room(x.device(), (given(a[2]) ? matrix : 0) + (normed ? matrix : 0) + (quantized ? eight_bytes(m, n, 1) : 0) + Room::padded(4 * m), 0);
  at::Tensor h = x, y;
  const void* r = nullptr;
  void* to = nullptr;
  int64_t ldr = 0;
  if (given(a[2])) {
    ldr = like(tensor(a[2]), x);
    r = tensor(a[2]).data_ptr();
    h = room.take({m, n}, x.scalar_type());
    to = h.data_ptr();
  }
  if (normed) y = room.take({m, n}, x.scalar_type());
  Eight e;
  if (quantized) e = eight_room(m, n, 1, room);
  const at::Tensor rstd = room.take({m}, at::kFloat);
  const int rc = slp_rmsnorm(x.data_ptr(), ldx, r, ldr, gamma, (float)number(a[3]), dt, side(m), side(n), to, n, address(y), n, e.at, e.ld, e.scales_at, e.lds,
                             (float*)rstd.data_ptr(), on.stream());
  return rc ? code(rc) : tuple({h, rstd, y, e.q, e.scales});
}

// dy, h, gamma, rstd, dh, gamma_grad
PyObject* rmsnorm_backward(PyObject* const* a) {
  const at::Tensor &dy = tensor(a[0]), &h = tensor(a[1]);
  const int64_t ldh = leading(h), lddy = like(dy, h), m = h.size(0), n = h.size(1);
  const int dt = dtype_of(h);
  const void* dh = nullptr;
  int64_t lddh = 0;
  if (given(a[4])) {
    lddh = like(tensor(a[4]), h);
    dh = tensor(a[4]).data_ptr();
  }
  require(given(a[3]), "rstd of the forward pass is wanted");
  const float *gamma = vector(a[2], n, h), *rstd = vector(a[3], m, h);
  const size_t size = slp_rmsnorm_backward_workspace_bytes(side(m), side(n));
  const On on(h.device());
  Room room(h.device(), Room::padded((size_t)(m * n) * (dt == SLP_BF16 ? 2 : 4)) + Room::padded(4 * n), size);
  const at::Tensor dx = room.take({m, n}, h.scalar_type());
  at::Tensor dgamma;
  if (truth(a[5])) dgamma = room.take({n}, at::kFloat);
  const at::Tensor work = room.work(size);
  const int rc = slp_rmsnorm_backward(dy.data_ptr(), lddy, h.data_ptr(), ldh, gamma, rstd, dh, lddh, dt, side(m), side(n), dx.data_ptr(), n, (float*)address(dgamma),
                                      address(work), size, on.stream());
  return rc ? code(rc) : tuple({dx, dgamma});
}

// What the two losses over a linear layer's classes share: the operands, the outputs and the workspace.
struct LossCall {
  const at::Tensor &x, &w;
  int64_t ldx, ldw, rows, dim, classes;
  int dt, dw_dt = 0;
  const float* bias;
  bool gradients, weight_gradients;
  at::Tensor loss, losses, lse, dx, dw, dbias, work;
  size_t size = 0;
  LossCall(PyObject* px, PyObject* pw, PyObject* pbias, bool grads, bool weight_grads)
      : x(tensor(px)), w(tensor(pw)), ldx(leading(x)), ldw(leading(w)), rows(x.size(0)), dim(x.size(1)), classes(w.size(0)), dt(dtype_of(x)), gradients(grads), weight_gradients(grads && weight_grads) {
    require(w.scalar_type() == x.scalar_type() && w.device() == x.device() && w.size(1) == dim, "weights of the rows' width, type and device are wanted");
    bias = vector(pbias, classes, x);
  }
  // top: entries of a distillation, 0 without.  dtype of the weights' gradient: SLP_F32, SLP_BF16, or None for the weights' own.
  void room(int64_t top, PyObject* dtype) {
    dw_dt = given(dtype) ? (int)integer(dtype) : dt;
    require(dw_dt == SLP_F32 || dw_dt == SLP_BF16, "float32 or bfloat16 is wanted");
    const bool b = weight_gradients && bias;
    size = slp_linear_loss_workspace_bytes(x.data_ptr(), ldx, w.data_ptr(), ldw, dt, side(rows), side(classes), side(dim), side(top),
                                           (gradients ? SLP_LOSS_DX : 0) | (weight_gradients ? SLP_LOSS_DW : 0) | (b ? SLP_LOSS_DBIAS : 0));
    const at::ScalarType type = dw_dt == SLP_BF16 ? at::kBFloat16 : at::kFloat;
    const size_t es = dt == SLP_BF16 ? 2 : 4;
    Room r(x.device(), 3 * Room::padded(4 * rows + 4) + (gradients ? Room::padded((size_t)(rows * dim) * es) : 0) +
                           (weight_gradients ? Room::padded((size_t)(classes * dim) * (dw_dt == SLP_BF16 ? 2 : 4)) : 0) + (b ? Room::padded(4 * classes) : 0), size);
    loss = r.take({}, at::kFloat);
    losses = r.take({rows}, at::kFloat);
    lse = r.take({rows}, at::kFloat);
    if (gradients) dx = r.take({rows, dim}, x.scalar_type());
    if (weight_gradients) dw = r.take({classes, dim}, type);
    if (b) dbias = r.take({classes}, at::kFloat);
    work = r.work(size);
  }
  PyObject* results() const { return tuple({loss, losses, lse, dx, dw, dbias}); }
};
int id_bytes(const at::Tensor& t, const at::Tensor& x) {
  require(t.device() == x.device() && (t.scalar_type() == at::kInt || t.scalar_type() == at::kLong), "class ids of int32 or int64 on the same device are wanted");
  return t.scalar_type() == at::kLong ? 8 : 4;
}

// x, w, targets, bias, gradients, weight_gradients, scale, dtype
PyObject* linear_cross_entropy(PyObject* const* a) {
  LossCall c(a[0], a[1], a[3], truth(a[4]), truth(a[5]));
  const at::Tensor& y = tensor(a[2]);
  const int bytes = id_bytes(y, c.x);
  require(y.is_contiguous() && y.dim() == 1 && y.numel() == c.rows, "a contiguous vector of one class id a row is wanted");
  const On on(c.x.device());
  c.room(0, a[7]);
  const int rc = slp_linear_cross_entropy(c.x.data_ptr(), c.ldx, c.w.data_ptr(), c.ldw, c.bias, c.dt, side(c.rows), side(c.classes), side(c.dim), y.data_ptr(), bytes, (float)number(a[6]),
                                          (float*)address(c.loss), (float*)address(c.losses), (float*)address(c.lse), address(c.dx), c.dim, address(c.dw), c.dim, c.dw_dt,
                                          (float*)address(c.dbias), address(c.work), c.size, on.stream());
  return rc ? code(rc) : c.results();
}

// x, w, top, classes, bias, temperature, gradients, weight_gradients, scale, dtype
PyObject* linear_distillation(PyObject* const* a) {
  LossCall c(a[0], a[1], a[4], truth(a[6]), truth(a[7]));
  const at::Tensor &top = tensor(a[2]), &ids = tensor(a[3]);
  const int64_t ldtop = leading(top), ldids = leading(ids), k = top.size(1);
  const int bytes = id_bytes(ids, c.x), top_dt = dtype_of(top);
  require(top.device() == c.x.device() && top.size(0) == c.rows && ids.sizes() == top.sizes(), "the teacher's logits and their classes, as many a row, are wanted");
  const On on(c.x.device());
  c.room(k, a[9]);
  const int rc = slp_linear_distillation(c.x.data_ptr(), c.ldx, c.w.data_ptr(), c.ldw, c.bias, c.dt, side(c.rows), side(c.classes), side(c.dim), top.data_ptr(), ldtop, top_dt, ids.data_ptr(),
                                         ldids, bytes, side(k), (float)number(a[5]), (float)number(a[8]), (float*)address(c.loss), (float*)address(c.losses), (float*)address(c.lse),
                                         address(c.dx), c.dim, address(c.dw), c.dim, c.dw_dt, (float*)address(c.dbias), address(c.work), c.size, on.stream());
  return rc ? code(rc) : c.results();
}

// Several tensors as the library takes them.  They are held until the call is queued: what an iterator makes has no other owner, and its memory would be
// given to the outputs and the workspace.
struct Tensors {
  THPObjectPtr held;
  std::vector<void*> at;
  std::vector<int64_t> counts;
  std::vector<int> dts;
  at::Device device = at::kCPU;
};
Tensors tensors(PyObject* list, const Tensors* as) {
  Tensors all;
  all.held = THPObjectPtr(PySequence_Tuple(list));
  if (!all.held) throw python_error();
  const Py_ssize_t n = PyTuple_GET_SIZE(all.held.get());
  require(n > 0, "at least one tensor is wanted");
  require(!as || as->at.size() == (size_t)n, "as many outputs as tensors are wanted");
  all.at.reserve((size_t)n);
  all.counts.reserve((size_t)n);
  all.dts.reserve((size_t)n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& t = tensor(PyTuple_GET_ITEM(all.held.get(), i));
    require(t.is_cuda() && t.is_contiguous(), "contiguous tensors on the device are wanted");
    if (i == 0) all.device = t.device();
    require(t.device() == all.device, "tensors on one device are wanted");
    all.at.push_back(t.data_ptr());
    all.counts.push_back(t.numel());
    all.dts.push_back(dtype_of(t));
    require(!as || (as->counts[i] == all.counts[i] && as->dts[i] == all.dts[i] && as->device == all.device), "outputs of the tensors' sizes and types are wanted");
  }
  return all;
}

// tensors
PyObject* gradient_norm(PyObject* const* a) {
  const Tensors in = tensors(a[0], nullptr);
  const int n = (int)in.at.size();
  const size_t size = slp_gradient_norm_workspace_bytes(n);
  const On on(in.device);
  Room room(in.device, Room::padded(4), size);
  const at::Tensor norm = room.take({}, at::kFloat), work = room.work(size);
  const int rc = slp_gradient_norm(in.at.data(), in.counts.data(), in.dts.data(), n, (float*)norm.data_ptr(), address(work), size, on.stream());
  if (rc) return code(rc);
  return wrapped(norm);
}

// tensors, max_norm, out
PyObject* clip_gradients(PyObject* const* a) {
  const Tensors in = tensors(a[0], nullptr);
  const int n = (int)in.at.size();
  Tensors out;
  if (given(a[2])) out = tensors(a[2], &in);
  const size_t size = slp_gradient_norm_workspace_bytes(n);
  const On on(in.device);
  Room room(in.device, Room::padded(4), size);
  const at::Tensor norm = room.take({}, at::kFloat), work = room.work(size);
  const int rc = slp_clip_gradients(in.at.data(), given(a[2]) ? out.at.data() : nullptr, in.counts.data(), in.dts.data(), n, (float)number(a[1]), (float*)norm.data_ptr(),
                                    address(work), size, on.stream());
  if (rc) return code(rc);
  return wrapped(norm);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    require(n == N, "wrong number of arguments");
    return F(args);
  } catch (const Refused& r) {
    PyErr_SetString(PyExc_AssertionError, r.what.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*F)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
  return {name, (PyCFunction)(void (*)())entry<F, N>, METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<quantize, 6>("quantize"),           method<product, 11>("product"), method<rmsnorm, 6>("rmsnorm"), method<rmsnorm_backward, 6>("rmsnorm_backward"),
                         method<gradient_norm, 1>("gradient_norm"), method<clip_gradients, 3>("clip_gradients"),
                         method<quantize_integers, 3>("quantize_integers"), method<product_integers, 8>("product_integers"),
                         method<linear_cross_entropy, 8>("linear_cross_entropy"), method<linear_distillation, 10>("linear_distillation"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
