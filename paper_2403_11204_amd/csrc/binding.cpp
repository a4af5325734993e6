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
                         method<gradient_norm, 1>("gradient_norm"), method<clip_gradients, 3>("clip_gradients"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
