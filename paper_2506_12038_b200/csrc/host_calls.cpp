// The calls of binding.py that a running program repeats, as a CPython module: arguments checked, outputs allocated and the
// C ABI called without going through ctypes and a Python-level tensor method per argument.  The kernels of one 4096 x 4096
// projection at one token take 8 us; the two calls it needs took 12.6 us on the host through ctypes (1.4 us a call for the
// argument conversion alone, the rest in tensor methods), which bounded every small case: 12.9 us a projection, 8.1 so (and a
// first pass over new buffers 35 instead of 49).  Failures are reported as the
// C ABI's status, an int, where a call returns tensors otherwise; binding.py turns it into LcdError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <vector>

#include "lcd.h"

namespace {

const at::Tensor* tensor_of(PyObject* o, const char* what) {
  if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
  PyErr_Format(PyExc_TypeError, "%s must be a torch.Tensor", what);
  return nullptr;
}
// A tensor's address; None: null.
bool address_of(PyObject* o, const char* what, void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o, what);
  if (!t) return false;
  *out = t->data_ptr();
  return true;
}
bool require(bool ok, const char* what) {
  if (!ok) PyErr_SetString(PyExc_AssertionError, what);
  return ok;
}
// The stream of a call: a torch stream object's, or the current one of the current device.  For its life a given stream is the
// current one, so that what the call allocates belongs to the stream that its kernels run on and is cleared there; outputs are
// recorded for the caller's stream as well, whose kernels will read them.
class CallStream {
 public:
  explicit CallStream(PyObject* o) : caller_(c10::cuda::getCurrentCUDAStream()), raw_(caller_.stream()) {
    if (o == Py_None) return;
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    void* given = h ? PyLong_AsVoidPtr(h) : nullptr;
    Py_XDECREF(h);
    failed_ = PyErr_Occurred() != nullptr;
    if (failed_ || given == raw_) return;
    raw_ = static_cast<cudaStream_t>(given);
    c10::cuda::setCurrentCUDAStream(c10::cuda::getStreamFromExternal(raw_, caller_.device_index()));
    other_ = true;
  }
  ~CallStream() {
    if (other_) c10::cuda::setCurrentCUDAStream(caller_);
  }
  CallStream(const CallStream&) = delete;
  CallStream& operator=(const CallStream&) = delete;
  bool ok() const { return !failed_; }
  void* raw() const { return raw_; }
  PyObject* output(const at::Tensor& t) const {
    if (other_) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), caller_);
    return THPVariable_Wrap(t);
  }

 private:
  c10::cuda::CUDAStream caller_;
  cudaStream_t raw_;
  bool failed_ = false, other_ = false;
};
bool count_args(Py_ssize_t have, Py_ssize_t want) {
  if (have != want) PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, have);
  return have == want;
}
template <typename Call>
lcd_status without_gil(Call&& call) {
  lcd_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return st;
}

// (x, inv_smooth, static_scale, act_idx, act_scale, act_bits, stream) -> (act_idx, act_scale) or a status
PyObject* smooth_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 7)) return nullptr;
  const at::Tensor* x = tensor_of(a[0], "x");
  if (!x || !require(x->is_cuda() && x->scalar_type() == at::kHalf && x->dim() == 2 && x->stride(1) == 1,
                     "x: CUDA fp16 [M, K] with unit column stride"))
    return nullptr;
  const int64_t M = x->size(0), K = x->size(1), K_pad = (K + 255) / 256 * 256;
  const long bits = PyLong_AsLong(a[5]);
  if ((bits == -1 && PyErr_Occurred()) || !require(bits == 4 || bits == 8, "act_bits: 4 or 8")) return nullptr;
  const at::ScalarType type = bits == 4 ? at::kByte : at::kChar;
  const CallStream stream(a[6]);
  if (!stream.ok()) return nullptr;
  at::Tensor idx, scale;
  if (a[3] == Py_None) idx = at::empty({M, bits == 4 ? K_pad / 2 : K_pad}, x->options().dtype(type));
  else if (const at::Tensor* t = tensor_of(a[3], "act_idx")) idx = *t;
  else return nullptr;
  if (!require(idx.scalar_type() == type, "act_idx: uint8 for 4-bit levels, int8 for 8-bit levels")) return nullptr;
  if (a[4] == Py_None) scale = at::empty({M}, x->options().dtype(at::kFloat));
  else if (const at::Tensor* t = tensor_of(a[4], "act_scale")) scale = *t;
  else return nullptr;
  void *inv, *fixed;
  if (!address_of(a[1], "inv_smooth", &inv) || !address_of(a[2], "static_scale", &fixed)) return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_smooth_quantize_act(x->data_ptr(), M, K, x->stride(0), static_cast<float*>(inv), static_cast<float*>(fixed),
                                   (int)bits, static_cast<uint8_t*>(idx.data_ptr()), static_cast<float*>(scale.data_ptr()), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  PyObject* o0 = a[3] == Py_None ? stream.output(idx) : Py_NewRef(a[3]);
  PyObject* o1 = a[4] == Py_None ? stream.output(scale) : Py_NewRef(a[4]);
  PyObject* out = o0 && o1 ? PyTuple_Pack(2, o0, o1) : nullptr;
  Py_XDECREF(o0);
  Py_XDECREF(o1);
  return out;
  END_HANDLE_TH_ERRORS
}

// (weights, header address, N, {(M, algo): workspace bytes}, act_idx, act_scale, y, algo, workspace, status_word, stream) -> y or a
// status; None: the table does not hold the size yet
PyObject* lut_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 11)) return nullptr;
  const at::Tensor *w = tensor_of(a[0], "weights"), *idx = w ? tensor_of(a[4], "act_idx") : nullptr;
  const at::Tensor* scale = idx ? tensor_of(a[5], "act_scale") : nullptr;
  if (!scale) return nullptr;
  void* header = PyLong_AsVoidPtr(a[1]);
  const int64_t N = PyLong_AsLongLong(a[2]);
  const long algo = PyLong_AsLong(a[7]);
  if (PyErr_Occurred()) return nullptr;
  if (!require(idx->dim() >= 1, "act_idx: [M, levels]")) return nullptr;
  const int64_t M = idx->size(0);
  size_t need = 0;
  {
    PyObject* key = Py_BuildValue("(LO)", (long long)M, a[7]);
    if (!key) return nullptr;
    PyObject* bytes = PyDict_GetItemWithError(a[3], key);
    Py_DECREF(key);
    if (!bytes) {
      if (PyErr_Occurred()) return nullptr;
      Py_RETURN_NONE;
    }
    need = PyLong_AsSize_t(bytes);
    if (PyErr_Occurred()) return nullptr;
  }
  const CallStream stream(a[10]);
  if (!stream.ok()) return nullptr;
  at::Tensor y, ws;
  if (a[6] == Py_None) y = at::empty({M, N}, idx->options().dtype(at::kFloat));
  else if (const at::Tensor* t = tensor_of(a[6], "y")) y = *t;
  else return nullptr;
  if (a[8] != Py_None) {
    const at::Tensor* t = tensor_of(a[8], "workspace");
    if (!t) return nullptr;
    ws = *t;
  }
  size_t have = ws.defined() ? (size_t)ws.numel() * ws.element_size() : 0;
  if (have < need) {
    ws = at::zeros({(int64_t)need}, idx->options().dtype(at::kByte));      // must start zero-filled
    have = need;
  }
  void* word;
  if (!address_of(a[9], "status_word", &word)) return nullptr;
  void* scratch = ws.defined() ? ws.data_ptr() : nullptr;
  const lcd_status st = without_gil([&] {
    const float* s = static_cast<const float*>(scale->data_ptr());
    float* out = static_cast<float*>(y.data_ptr());
    int32_t* flag = static_cast<int32_t*>(word);
    return idx->scalar_type() == at::kChar
               ? lcd_lut_linear_act8(w->data_ptr(), header, static_cast<const int8_t*>(idx->data_ptr()), s, M, out, y.stride(0),
                                     (lcd_algo)algo, scratch, have, flag, stream.raw())
               : lcd_lut_linear(w->data_ptr(), header, static_cast<const uint8_t*>(idx->data_ptr()), s, M, out, y.stride(0),
                                (lcd_algo)algo, scratch, have, flag, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return a[6] == Py_None ? stream.output(y) : Py_NewRef(a[6]);
  END_HANDLE_TH_ERRORS
}

// (problem array address, count, act_bits, stream) -> status
PyObject* act_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 4)) return nullptr;
  void* arr = PyLong_AsVoidPtr(a[0]);
  const int count = (int)PyLong_AsLong(a[1]), bits = (int)PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  const CallStream stream(a[3]);
  if (!stream.ok()) return nullptr;
  return PyLong_FromLong((long)without_gil(
      [&] { return lcd_smooth_quantize_act_batch(static_cast<const lcd_act_problem*>(arr), count, bits, stream.raw()); }));
  END_HANDLE_TH_ERRORS
}

// (form, problem array address, count, algo, workspace, status_word, stream) -> status; form 0: fused, 1: stored 4-bit levels,
// 2: stored 8-bit levels
PyObject* linear_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 7)) return nullptr;
  const long form = PyLong_AsLong(a[0]);
  void *arr = PyLong_AsVoidPtr(a[1]), *word;
  const int count = (int)PyLong_AsLong(a[2]);
  const lcd_algo algo = (lcd_algo)PyLong_AsLong(a[3]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor* ws = tensor_of(a[4], "workspace");
  if (!ws || !address_of(a[5], "status_word", &word)) return nullptr;
  const CallStream stream(a[6]);
  if (!stream.ok()) return nullptr;
  void* scratch = ws->data_ptr();
  const size_t bytes = (size_t)ws->numel();
  return PyLong_FromLong((long)without_gil([&] {
    int32_t* flag = static_cast<int32_t*>(word);
    if (form == 0) return lcd_linear_fused_batch(static_cast<const lcd_fused_problem*>(arr), count, algo, scratch, bytes, flag, stream.raw());
    const lcd_linear_problem* p = static_cast<const lcd_linear_problem*>(arr);
    return form == 1 ? lcd_lut_linear_batch(p, count, algo, scratch, bytes, flag, stream.raw())
                     : lcd_lut_linear_batch_act8(p, count, algo, scratch, bytes, flag, stream.raw());
  }));
  END_HANDLE_TH_ERRORS
}

// (idx, codebook, delta_w, new_idx, delta_c, counts, stream) -> (new_idx, delta_c, counts) or a status
PyObject* reclassify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 7)) return nullptr;
  const at::Tensor *idx = tensor_of(a[0], "idx"), *cb = idx ? tensor_of(a[1], "codebook") : nullptr;
  const at::Tensor* dw = cb ? tensor_of(a[2], "delta_w") : nullptr;
  if (!dw || !require(idx->scalar_type() == at::kByte && cb->scalar_type() == at::kHalf && dw->scalar_type() == at::kFloat,
                      "idx uint8, codebook fp16, delta_w fp32") ||
      !require(idx->dim() == 2 && cb->dim() == 2 && dw->dim() == 2 && idx->is_contiguous() && cb->is_contiguous() &&
                   dw->stride(1) == 1, "contiguous [N, K], [N, C] and rows of delta_w"))
    return nullptr;
  const int64_t N = idx->size(0), K = idx->size(1), C = cb->size(1);
  const CallStream stream(a[6]);
  if (!stream.ok()) return nullptr;
  at::Tensor out[3];
  if (a[3] == Py_None) {
    out[0] = at::empty_like(*idx);
    out[1] = at::empty({N, C}, idx->options().dtype(at::kDouble));
    out[2] = at::empty({N, C}, idx->options().dtype(at::kInt));
  } else {
    for (int i = 0; i < 3; ++i) {
      const at::Tensor* t = tensor_of(a[3 + i], "out");
      if (!t) return nullptr;
      out[i] = *t;
    }
    if (!require(out[0].scalar_type() == at::kByte && out[1].scalar_type() == at::kDouble && out[2].scalar_type() == at::kInt,
                 "out: uint8, fp64, int32") ||
        !require(out[0].sizes() == idx->sizes() && out[1].sizes() == cb->sizes() && out[2].sizes() == cb->sizes(),
                 "out: [N, K], [N, C], [N, C]"))
      return nullptr;
  }
  const lcd_status st = without_gil([&] {
    return lcd_reclassify(static_cast<const uint8_t*>(idx->data_ptr()), static_cast<const uint16_t*>(cb->data_ptr()),
                          static_cast<const float*>(dw->data_ptr()), N, K, dw->stride(0), (int)C,
                          static_cast<uint8_t*>(out[0].data_ptr()), static_cast<double*>(out[1].data_ptr()),
                          static_cast<int32_t*>(out[2].data_ptr()), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  if (a[3] != Py_None) return PyTuple_Pack(3, a[3], a[4], a[5]);
  PyObject* r = PyTuple_New(3);
  for (int i = 0; r && i < 3; ++i) {
    PyObject* o = stream.output(out[i]);
    if (!o) Py_CLEAR(r);
    else PyTuple_SET_ITEM(r, i, o);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// (x, wmax, alphas, stream) -> (best, mse, inv_smooth) or a status
PyObject* smoothing_search(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 4)) return nullptr;
  const at::Tensor *x = tensor_of(a[0], "x"), *wmax = x ? tensor_of(a[1], "wmax") : nullptr;
  if (!wmax || !require(x->is_cuda() && x->scalar_type() == at::kHalf && x->dim() == 2 && x->stride(1) == 1,
                        "x: CUDA fp16 [T, K] with unit column stride"))
    return nullptr;
  PyObject* list = PySequence_Fast(a[2], "alphas: a sequence of floats");
  if (!list) return nullptr;
  std::vector<float> alphas((size_t)PySequence_Fast_GET_SIZE(list));
  for (size_t i = 0; i < alphas.size(); ++i) alphas[i] = (float)PyFloat_AsDouble(PySequence_Fast_GET_ITEM(list, (Py_ssize_t)i));
  Py_DECREF(list);
  if (PyErr_Occurred()) return nullptr;
  const int64_t T = x->size(0), K = x->size(1);
  const int G = (int)alphas.size();
  size_t need = 0;
  const lcd_status sized = lcd_smoothing_search_workspace_bytes(T, K, G, &need);
  if (sized != LCD_OK) return PyLong_FromLong((long)sized);
  const CallStream stream(a[3]);
  if (!stream.ok()) return nullptr;
  const at::Tensor ws = at::empty({(int64_t)need}, x->options().dtype(at::kByte));
  const at::Tensor mse = at::empty({G}, x->options().dtype(at::kDouble)), best = at::empty({1}, x->options().dtype(at::kInt)),
                   inv = at::empty({K}, x->options().dtype(at::kFloat));
  const lcd_status st = without_gil([&] {
    return lcd_smoothing_search(x->data_ptr(), T, K, x->stride(0), static_cast<const float*>(wmax->data_ptr()), alphas.data(), G,
                                ws.data_ptr(), need, static_cast<double*>(mse.data_ptr()), static_cast<int32_t*>(best.data_ptr()),
                                static_cast<float*>(inv.data_ptr()), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  PyObject *o0 = stream.output(best), *o1 = stream.output(mse), *o2 = stream.output(inv);
  PyObject* out = o0 && o1 && o2 ? PyTuple_Pack(3, o0, o1, o2) : nullptr;
  Py_XDECREF(o0);
  Py_XDECREF(o1);
  Py_XDECREF(o2);
  return out;
  END_HANDLE_TH_ERRORS
}

// ---- microscaled 4-bit floating point and distillation.  These run on their first tensor's device, whichever is current, and
// every tensor has to lie there.
// A new tensor, without the dispatcher (0.5 us each, of a call of 5).
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Device& device) {
  return at::detail::empty_cuda(shape, type, device, std::nullopt);
}
bool type_of(at::ScalarType t, lcd_dtype* out) {
  if (t == at::kFloat) *out = LCD_DTYPE_F32;
  else if (t == at::kHalf) *out = LCD_DTYPE_F16;
  else if (t == at::kBFloat16) *out = LCD_DTYPE_BF16;
  else return false;
  return true;
}
// A matrix of fp32, fp16 or bf16 with unit column stride.
bool dense(const at::Tensor& t, lcd_dtype* type) {
  return t.is_cuda() && t.dim() == 2 && type_of(t.scalar_type(), type) && (t.stride(1) == 1 || t.size(1) == 1);
}
// Elements from a row to the next.  A single row's stride is whatever its tensor was cut from: any that holds the row will do.
int64_t row_stride(const at::Tensor& t, int64_t multiple = 1) {
  return t.size(0) > 1 ? t.stride(0) : (t.size(1) + multiple - 1) / multiple * multiple;
}
bool bytes_of(const at::Tensor& t, const at::Device& device, int64_t rows, int64_t columns) {
  return t.device() == device && t.scalar_type() == at::kByte && t.dim() == 2 && t.size(0) == rows && t.size(1) == columns &&
         (t.stride(1) == 1 || columns == 1);
}
// An fp32 vector of n values, or none.
bool vector_of(PyObject* o, const char* what, const at::Device& device, int64_t n, const char* expected, const float** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o, what);
  if (!t || !require(t->device() == device && t->scalar_type() == at::kFloat && t->numel() == n && t->is_contiguous(), expected)) return false;
  *out = static_cast<const float*>(t->data_ptr());
  return true;
}
bool status_word_of(PyObject* o, const at::Device& device, int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o, "status_word");
  if (!t || !require(t->device() == device && t->scalar_type() == at::kInt && t->numel() >= 1, "status_word: int32 on the same device")) return false;
  *out = static_cast<int32_t*>(t->data_ptr());
  return true;
}
// A dtype argument (torch.float32, float16, bfloat16).
bool dtype_of(PyObject* o, at::ScalarType* out) {
  lcd_dtype t;
  if (!require(THPDtype_Check(o), "dtype: a torch.dtype")) return false;
  *out = reinterpret_cast<THPDtype*>(o)->scalar_type;
  return require(type_of(*out, &t), "dtype: torch.float32, torch.float16 or torch.bfloat16");
}
// The given tensor of that shape, or a new one.
bool output_of(PyObject* o, const char* what, at::IntArrayRef shape, at::ScalarType type, const at::Device& device, const char* expected,
               at::Tensor* out) {
  if (o == Py_None) {
    *out = fresh(shape, type, device);
    return true;
  }
  const at::Tensor* t = tensor_of(o, what);
  if (!t || !require(t->device() == device && t->scalar_type() == type && t->sizes() == shape &&
                         (t->dim() == 0 || t->stride(-1) == 1 || t->size(-1) == 1), expected))
    return false;
  *out = *t;
  return true;
}
// A given output is returned as it came.
PyObject* returned(const CallStream& stream, PyObject* given, const at::Tensor& t) {
  return given == Py_None ? stream.output(t) : Py_NewRef(given);
}
PyObject* pack(std::initializer_list<PyObject*> items) {     // steals the references
  bool all = true;
  for (PyObject* o : items) all = all && o;
  PyObject* r = all ? PyTuple_New((Py_ssize_t)items.size()) : nullptr;
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (r) PyTuple_SET_ITEM(r, i++, o);
    else Py_XDECREF(o);
  }
  return r;
}

// (x, inv_smooth, codes, scales, stream) -> (codes, scales) or a status
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 5)) return nullptr;
  const at::Tensor* x = tensor_of(a[0], "x");
  lcd_dtype type;
  if (!x || !require(dense(*x, &type), "x: CUDA fp32, fp16 or bf16 [M, K] with unit column stride")) return nullptr;
  const c10::cuda::CUDAGuard on(x->device());
  const int64_t M = x->size(0), K = x->size(1), blocks = (K + 31) / 32;
  const float* inv;
  if (!vector_of(a[1], "inv_smooth", x->device(), K, "inv_smooth: fp32 [K] on x's device", &inv)) return nullptr;
  const CallStream stream(a[4]);
  if (!stream.ok()) return nullptr;
  at::Tensor codes, scales;
  if (!output_of(a[2], "codes", {M, 16 * blocks}, at::kByte, x->device(), "codes: uint8 [M, 16 * ceil(K / 32)]", &codes)) return nullptr;
  if (a[3] == Py_None) scales = at::detail::empty_strided_cuda({M, blocks}, {(blocks + 15) / 16 * 16, 1}, at::kByte, x->device());
  else if (!output_of(a[3], "scales", {M, blocks}, at::kByte, x->device(), "scales: uint8 [M, ceil(K / 32)]", &scales)) return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_mx_quantize(x->data_ptr(), type, M, K, row_stride(*x), inv, static_cast<uint8_t*>(codes.data_ptr()), row_stride(codes),
                           static_cast<uint8_t*>(scales.data_ptr()), row_stride(scales, 16), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return pack({returned(stream, a[2], codes), returned(stream, a[3], scales)});
  END_HANDLE_TH_ERRORS
}

// (codes, scales, K or None, out, dtype, stream) -> out or a status
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 6)) return nullptr;
  const at::Tensor *codes = tensor_of(a[0], "codes"), *scales = codes ? tensor_of(a[1], "scales") : nullptr;
  if (!scales || !require(codes->is_cuda() && codes->dim() == 2 && codes->size(1) % 16 == 0, "codes: CUDA uint8 [M, 16 * blocks]")) return nullptr;
  const int64_t M = codes->size(0), blocks = codes->size(1) / 16;
  const int64_t K = a[2] == Py_None ? 32 * blocks : PyLong_AsLongLong(a[2]);
  at::ScalarType type;
  if (PyErr_Occurred() || !dtype_of(a[4], &type)) return nullptr;
  if (!require(bytes_of(*codes, codes->device(), M, 16 * blocks) && bytes_of(*scales, codes->device(), M, blocks),
               "codes: uint8 [M, 16 * blocks], scales: uint8 [M, blocks], on one device") ||
      !require(K >= 1 && (K + 31) / 32 == blocks, "K: 32 * blocks, or up to 31 less"))
    return nullptr;
  const c10::cuda::CUDAGuard on(codes->device());
  const CallStream stream(a[5]);
  if (!stream.ok()) return nullptr;
  at::Tensor out;
  if (a[3] != Py_None) {
    const at::Tensor* t = tensor_of(a[3], "out");
    if (!t) return nullptr;
    type = t->scalar_type();
  }
  lcd_dtype kind;
  if (!require(type_of(type, &kind), "out: fp32, fp16 or bf16") ||
      !output_of(a[3], "out", {M, K}, type, codes->device(), "out: [M, K] with unit column stride on the codes' device", &out))
    return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_mx_dequantize(static_cast<const uint8_t*>(codes->data_ptr()), row_stride(*codes), static_cast<const uint8_t*>(scales->data_ptr()),
                             row_stride(*scales, 16), M, K, out.data_ptr(), kind, row_stride(out), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return returned(stream, a[3], out);
  END_HANDLE_TH_ERRORS
}

// (fused, w_codes, w_scales, x or x_codes, inv_smooth or x_scales, y, dtype, workspace, status_word, stream) -> y or a status
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 10)) return nullptr;
  const bool fused = PyObject_IsTrue(a[0]) == 1;
  const at::Tensor *wc = tensor_of(a[1], "w_codes"), *ws = wc ? tensor_of(a[2], "w_scales") : nullptr;
  const at::Tensor* x = ws ? tensor_of(a[3], fused ? "x" : "x_codes") : nullptr;
  if (!x || !require(wc->is_cuda() && wc->dim() == 2 && wc->size(1) % 16 == 0, "w_codes: CUDA uint8 [N, 16 * blocks]")) return nullptr;
  const at::Device device = wc->device();
  const int64_t N = wc->size(0), blocks = wc->size(1) / 16;
  if (!require(bytes_of(*wc, device, N, 16 * blocks) && bytes_of(*ws, device, N, blocks),
               "w_codes: uint8 [N, 16 * blocks], w_scales: uint8 [N, blocks], on one device") ||
      !require(x->dim() == 2 && x->device() == device, fused ? "x: [M, K] on the weights' device" : "x_codes: [M, 16 * blocks] on the weights' device"))
    return nullptr;
  const int64_t M = x->size(0);
  int64_t K = 32 * blocks;
  lcd_dtype x_type = LCD_DTYPE_F32, y_type;
  const at::Tensor* xs = nullptr;
  const float* inv = nullptr;
  if (fused) {
    K = x->size(1);
    if (!require(dense(*x, &x_type), "x: CUDA fp32, fp16 or bf16 [M, K] with unit column stride") ||
        !require((K + 31) / 32 == blocks, "x: [M, K], K being 32 * blocks of the weights, or up to 31 less") ||
        !vector_of(a[4], "inv_smooth", device, K, "inv_smooth: fp32 [K] on x's device", &inv))
      return nullptr;
  } else {
    xs = tensor_of(a[4], "x_scales");
    if (!xs || !require(bytes_of(*x, device, M, 16 * blocks) && bytes_of(*xs, device, M, blocks),
                        "x_codes: uint8 [M, 16 * blocks], x_scales: uint8 [M, blocks], blocks as the weights'"))
      return nullptr;
  }
  at::ScalarType type;
  if (!dtype_of(a[6], &type)) return nullptr;
  int32_t* word;
  if (!status_word_of(a[8], device, &word)) return nullptr;
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[9]);
  if (!stream.ok()) return nullptr;
  if (a[5] != Py_None) {
    const at::Tensor* t = tensor_of(a[5], "y");
    if (!t) return nullptr;
    type = t->scalar_type();
  }
  at::Tensor y, space;
  if (!require(type_of(type, &y_type), "y: fp32, fp16 or bf16") ||
      !output_of(a[5], "y", {M, N}, type, device, "y: [M, N] with unit column stride on the weights' device", &y))
    return nullptr;
  size_t have = 0;
  if (fused) {
    size_t need = 0;
    const lcd_status sized = lcd_mx_linear_fused_workspace_bytes(M, K, &need);
    if (sized != LCD_OK) return PyLong_FromLong((long)sized);
    if (a[7] == Py_None) {
      if (need > 0) space = fresh({(int64_t)need}, at::kByte, device);
    } else {
      const at::Tensor* t = tensor_of(a[7], "workspace");
      if (!t || !require(t->device() == device && t->is_contiguous(), "workspace: contiguous, on the weights' device")) return nullptr;
      space = *t;
    }
    have = space.defined() ? (size_t)space.numel() * space.element_size() : 0;
  }
  const lcd_status st = without_gil([&] {
    const uint8_t *c = static_cast<const uint8_t*>(wc->data_ptr()), *s = static_cast<const uint8_t*>(ws->data_ptr());
    const int64_t ldc = row_stride(*wc), lds = row_stride(*ws, 16), ldy = row_stride(y);
    if (fused)
      return lcd_mx_linear_fused(c, ldc, s, lds, N, K, x->data_ptr(), x_type, row_stride(*x), inv, M, y.data_ptr(), y_type, ldy,
                                 have ? space.data_ptr() : nullptr, have, word, stream.raw());
    return lcd_mx_linear(c, ldc, s, lds, N, K, static_cast<const uint8_t*>(x->data_ptr()), row_stride(*x),
                         static_cast<const uint8_t*>(xs->data_ptr()), row_stride(*xs, 16), M, y.data_ptr(), y_type, ldy, word, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return returned(stream, a[5], y);
  END_HANDLE_TH_ERRORS
}

// (logits, teacher_idx, teacher_logits, temperature, teacher_lse, weight, stats in or None, loss, stats out (None, True: a new one),
//  dlogits (None, True: a new one), stream) -> (loss, stats or None, dlogits or None), or a status.  With stats in: the gradient alone.
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 11)) return nullptr;
  const at::Tensor *z = tensor_of(a[0], "logits"), *idx = z ? tensor_of(a[1], "teacher_idx") : nullptr;
  const at::Tensor* top = idx ? tensor_of(a[2], "teacher_logits") : nullptr;
  lcd_dtype type, top_type;
  if (!top || !require(dense(*z, &type), "logits: CUDA fp32, fp16 or bf16 [T, V] with unit column stride")) return nullptr;
  const at::Device device = z->device();
  const int64_t T = z->size(0), V = z->size(1);
  if (!require(dense(*top, &top_type) && top->device() == device && top->size(0) == T,
               "teacher_logits: fp32, fp16 or bf16 [T, k] with unit column stride on the logits' device"))
    return nullptr;
  const int64_t k = top->size(1);
  if (!require(idx->device() == device && (idx->scalar_type() == at::kInt || idx->scalar_type() == at::kLong) && idx->dim() == 2 &&
                   idx->size(0) == T && idx->size(1) == k && (idx->stride(1) == 1 || k == 1),
               "teacher_idx: int32 or int64 [T, k] with unit column stride on the logits' device"))
    return nullptr;
  const double tau = PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) return nullptr;
  const float *lse, *weight;
  if (!vector_of(a[4], "teacher_lse", device, T, "teacher_lse: fp32 [T] on the logits' device", &lse) ||
      !vector_of(a[5], "weight", device, T, "weight: fp32 [T] on the logits' device", &weight))
    return nullptr;
  const bool grad_only = a[6] != Py_None;
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[10]);
  if (!stream.ok()) return nullptr;
  PyObject *want_stats = a[8] == Py_True ? Py_None : a[8], *want_grad = a[9] == Py_True ? Py_None : a[9];   // None from here: a new one
  const bool has_stats = grad_only || a[8] != Py_None, has_grad = a[9] != Py_None;
  at::Tensor loss, stats, d;
  if (!grad_only && (!output_of(a[7], "loss", {T}, at::kFloat, device, "loss: fp32 [T] on the logits' device", &loss) ||
                     !require(loss.is_contiguous(), "loss: contiguous")))
    return nullptr;
  if (has_stats && (!output_of(grad_only ? a[6] : want_stats, "stats", {T, 2}, at::kFloat, device, "stats: fp32 [T, 2] on the logits' device", &stats) ||
                    !require(stats.is_contiguous(), "stats: contiguous")))
    return nullptr;
  if (has_grad && !output_of(want_grad, "dlogits", {T, V}, z->scalar_type(), device, "dlogits: as the logits, with unit column stride", &d)) return nullptr;
  const lcd_status st = without_gil([&] {
    void* grads = has_grad ? d.data_ptr() : nullptr;
    const int64_t ldd = has_grad ? row_stride(d) : 0;
    float* state = has_stats ? static_cast<float*>(stats.data_ptr()) : nullptr;
    const int width = idx->scalar_type() == at::kInt ? 4 : 8;
    if (grad_only)
      return lcd_distill_grad(z->data_ptr(), type, T, V, row_stride(*z), idx->data_ptr(), width, row_stride(*idx), top->data_ptr(), top_type,
                              row_stride(*top), k, (float)tau, lse, weight, state, grads, ldd, stream.raw());
    return lcd_distill_loss(z->data_ptr(), type, T, V, row_stride(*z), idx->data_ptr(), width, row_stride(*idx), top->data_ptr(), top_type,
                            row_stride(*top), k, (float)tau, lse, weight, static_cast<float*>(loss.data_ptr()), state, grads, ldd, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return pack({grad_only ? Py_NewRef(Py_None) : returned(stream, a[7], loss),
               grad_only || !has_stats ? Py_NewRef(Py_None) : returned(stream, want_stats, stats),
               has_grad ? returned(stream, want_grad, d) : Py_NewRef(Py_None)});
  END_HANDLE_TH_ERRORS
}

// ---- rows that go to different weights
// The plan's three tensors: int32, contiguous, on one device.
bool plan_of(PyObject* const* a, const at::Device& device, int64_t* G, lcd_row_groups* out) {
  const at::Tensor *order = tensor_of(a[0], "order"), *groups = order ? tensor_of(a[1], "groups") : nullptr;
  const at::Tensor* offsets = groups ? tensor_of(a[2], "offsets") : nullptr;
  if (!offsets) return false;
  for (const at::Tensor* t : {order, groups, offsets})
    if (!require(t->device() == device && t->scalar_type() == at::kInt && t->dim() == 1 && t->is_contiguous(),
                 "rows: int32 order, groups and offsets, contiguous, on the same device as the other arguments"))
      return false;
  if (!require(groups->size(0) == order->size(0) && offsets->size(0) >= 2, "rows: as many groups as rows, an offset more than groups")) return false;
  *G = offsets->size(0) - 1;
  *out = {static_cast<const int32_t*>(order->data_ptr()), static_cast<const int32_t*>(groups->data_ptr()),
          static_cast<const int32_t*>(offsets->data_ptr()), order->size(0)};
  return true;
}
// A given workspace (contiguous, on the device) or a new one.
bool workspace_of(PyObject* o, size_t need, const at::Device& device, at::Tensor* space, size_t* have) {
  if (o == Py_None) {
    *space = fresh({(int64_t)need}, at::kByte, device);
  } else {
    const at::Tensor* t = tensor_of(o, "workspace");
    if (!t || !require(t->device() == device && t->is_contiguous(), "workspace: contiguous, on the same device")) return false;
    *space = *t;
  }
  *have = (size_t)space->numel() * space->element_size();
  return true;
}

// (group, G, order, groups, offsets, stream) -> (order, groups, offsets) or a status
PyObject* group_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 6)) return nullptr;
  const at::Tensor* group = tensor_of(a[0], "group");
  if (!group || !require(group->is_cuda() && group->is_contiguous() && (group->scalar_type() == at::kInt || group->scalar_type() == at::kLong),
                         "group: contiguous CUDA int32 or int64"))
    return nullptr;
  const int64_t G = PyLong_AsLongLong(a[1]), count = group->numel();
  if (PyErr_Occurred()) return nullptr;
  const at::Device device = group->device();
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[5]);
  if (!stream.ok()) return nullptr;
  if (count < 1 || G < 1) return PyLong_FromLong((long)LCD_ERR_INVALID_ARG);
  if (G > 1024 || count > (1ll << 30)) return PyLong_FromLong((long)(G > 1024 ? LCD_ERR_UNSUPPORTED : LCD_ERR_INVALID_ARG));
  at::Tensor order, groups, offsets;
  if (!output_of(a[2], "order", {count}, at::kInt, device, "order: int32 [rows] on group's device", &order) ||
      !output_of(a[3], "groups", {count}, at::kInt, device, "groups: int32 [rows] on group's device", &groups) ||
      !output_of(a[4], "offsets", {G + 1}, at::kInt, device, "offsets: int32 [G + 1] on group's device", &offsets) ||
      !require(order.is_contiguous() && groups.is_contiguous() && offsets.is_contiguous(), "order, groups, offsets: contiguous"))
    return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_group_rows(group->data_ptr(), group->scalar_type() == at::kInt ? 4 : 8, count, G, static_cast<int32_t*>(order.data_ptr()),
                          static_cast<int32_t*>(groups.data_ptr()), static_cast<int32_t*>(offsets.data_ptr()), stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return pack({returned(stream, a[2], order), returned(stream, a[3], groups), returned(stream, a[4], offsets)});
  END_HANDLE_TH_ERRORS
}

// (w_codes, w_scales, x, order, groups, offsets, inv_smooth, y, dtype, workspace, status_word, stream) -> y or a status
PyObject* mx_linear_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 12)) return nullptr;
  const at::Tensor *wc = tensor_of(a[0], "w_codes"), *ws = wc ? tensor_of(a[1], "w_scales") : nullptr, *x = ws ? tensor_of(a[2], "x") : nullptr;
  if (!x || !require(wc->is_cuda() && wc->scalar_type() == at::kByte && wc->dim() == 3 && wc->size(2) % 16 == 0 && wc->size(2) > 0 && wc->stride(2) == 1,
                     "w_codes: CUDA uint8 [G, N, 16 * blocks]"))
    return nullptr;
  const at::Device device = wc->device();
  const int64_t G = wc->size(0), N = wc->size(1), blocks = wc->size(2) / 16;
  if (!require(ws->device() == device && ws->scalar_type() == at::kByte && ws->dim() == 3 && ws->size(0) == G && ws->size(1) == N &&
                   ws->size(2) == blocks && (ws->stride(2) == 1 || blocks == 1),
               "w_scales: uint8 [G, N, blocks] on the codes' device"))
    return nullptr;
  lcd_dtype x_type, y_type;
  if (!require(dense(*x, &x_type) && x->device() == device, "x: fp32, fp16 or bf16 [T, K] with unit column stride on the weights' device")) return nullptr;
  const int64_t T = x->size(0), K = x->size(1);
  int64_t groups;
  lcd_row_groups rows;
  const float* inv;
  int32_t* word;
  at::ScalarType type;
  if (!require((K + 31) / 32 == blocks, "x: [T, K], K being 32 * blocks of the weights, or up to 31 less") || !plan_of(a + 3, device, &groups, &rows) ||
      !require(groups == G, "rows: a plan of as many groups as there are experts") ||
      !require(T > 0 && rows.count % T == 0, "rows: a multiple of x's rows") ||
      !vector_of(a[6], "inv_smooth", device, K, "inv_smooth: fp32 [K] on x's device", &inv) || !dtype_of(a[8], &type) ||
      !status_word_of(a[10], device, &word))
    return nullptr;
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[11]);
  if (!stream.ok()) return nullptr;
  if (a[7] != Py_None) {
    const at::Tensor* t = tensor_of(a[7], "y");
    if (!t) return nullptr;
    type = t->scalar_type();
  }
  size_t need = 0, have = 0;
  const lcd_status sized = lcd_mx_linear_grouped_workspace_bytes(rows.count, K, &need);
  if (sized != LCD_OK) return PyLong_FromLong((long)sized);
  at::Tensor y, space;
  if (!require(type_of(type, &y_type), "y: fp32, fp16 or bf16") ||
      !output_of(a[7], "y", {rows.count, N}, type, device, "y: [rows, N] with unit column stride on the weights' device", &y) ||
      !workspace_of(a[9], need, device, &space, &have))
    return nullptr;
  const lcd_status st = without_gil([&] {
    const int64_t ldc = N > 1 ? wc->stride(1) : 16 * blocks, lds = N > 1 ? ws->stride(1) : (blocks + 15) / 16 * 16;
    return lcd_mx_linear_grouped(static_cast<const uint8_t*>(wc->data_ptr()), ldc, wc->stride(0), static_cast<const uint8_t*>(ws->data_ptr()), lds,
                                 ws->stride(0), G, N, K, x->data_ptr(), x_type, T, row_stride(*x), inv, &rows, y.data_ptr(), y_type, row_stride(y),
                                 have ? space.data_ptr() : nullptr, have, word, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return returned(stream, a[7], y);
  END_HANDLE_TH_ERRORS
}

// The adapters' matrices and factors.
bool adapters_of(PyObject* a, PyObject* b, PyObject* scale, lcd_adapter_weights* w, at::Device* device) {
  const at::Tensor *ta = tensor_of(a, "a"), *tb = ta ? tensor_of(b, "b") : nullptr;
  if (!tb || !require(ta->is_cuda() && ta->dim() == 3 && type_of(ta->scalar_type(), &w->type) && (ta->stride(2) == 1 || ta->size(2) == 1),
                      "a: CUDA fp32, fp16 or bf16 [G, rank, K] with unit column stride") ||
      !require(tb->device() == ta->device() && tb->dim() == 3 && tb->scalar_type() == ta->scalar_type() && (tb->stride(2) == 1 || tb->size(2) == 1) &&
                   tb->size(0) == ta->size(0) && tb->size(2) == ta->size(1),
               "b: [G, N, rank] of a's type, with unit column stride, on a's device"))
    return false;
  *device = ta->device();
  w->a = ta->data_ptr();
  w->b = tb->data_ptr();
  w->G = ta->size(0);
  w->rank = ta->size(1);
  w->K = ta->size(2);
  w->N = tb->size(1);
  w->lda = w->rank > 1 ? ta->stride(1) : w->K;
  w->ldb = w->N > 1 ? tb->stride(1) : w->rank;
  w->adapter_a = ta->stride(0);
  w->adapter_b = tb->stride(0);
  return vector_of(scale, "scale", *device, w->G, "scale: fp32 [G] on the adapters' device", &w->scale);
}
bool rows_of_x(const at::Tensor* x, const at::Device& device, int64_t count, int64_t columns, lcd_dtype* type, const char* expected) {
  return x && require(dense(*x, type) && x->device() == device && x->size(0) == count && x->size(1) == columns, expected);
}

// (x, a, b, order, groups, offsets, base, y, scale, dtype or None, t (None, True: a new one), workspace, status_word, stream) -> (y, t or None) or a status
PyObject* adapters(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 14)) return nullptr;
  lcd_adapter_weights w = {};
  int32_t* word;
  at::Device device(at::kCPU);
  int64_t groups;
  lcd_row_groups rows;
  lcd_dtype x_type, y_type, base_type;
  if (!adapters_of(a[1], a[2], a[8], &w, &device) || !plan_of(a + 3, device, &groups, &rows) || !status_word_of(a[12], device, &word) ||
      !require(groups == w.G, "rows: a plan of as many groups as there are adapters"))
    return nullptr;
  const at::Tensor *x = tensor_of(a[0], "x"), *base = nullptr;
  if (!rows_of_x(x, device, rows.count, w.K, &x_type, "x: fp32, fp16 or bf16 [rows, K] with unit column stride on the adapters' device")) return nullptr;
  at::ScalarType type = x->scalar_type();
  if (a[9] != Py_None && !dtype_of(a[9], &type)) return nullptr;
  if (a[6] != Py_None) {
    base = tensor_of(a[6], "base");
    if (!rows_of_x(base, device, rows.count, w.N, &base_type, "base: fp32, fp16 or bf16 [rows, N] with unit column stride on the adapters' device") ||
        !require(a[9] == Py_None || base->scalar_type() == type, "dtype: base's"))
      return nullptr;
    type = base->scalar_type();
  } else if (a[7] != Py_None && a[9] == Py_None) {
    const at::Tensor* t = tensor_of(a[7], "y");
    if (!t) return nullptr;
    type = t->scalar_type();
  }
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[13]);
  if (!stream.ok()) return nullptr;
  size_t need = 0, have = 0;
  const lcd_status sized = lcd_adapters_workspace_bytes(rows.count, w.rank, &need);
  if (sized != LCD_OK) return PyLong_FromLong((long)sized);
  PyObject* want_t = a[10] == Py_True ? Py_None : a[10];
  const bool has_t = a[10] != Py_None;
  at::Tensor y, t, space;
  if (!require(type_of(type, &y_type), "y: fp32, fp16 or bf16") ||
      !output_of(a[7], "y", {rows.count, w.N}, type, device, "y: [rows, N] of base's type, with unit column stride, on the adapters' device", &y) ||
      (has_t && !output_of(want_t, "t", {rows.count, w.rank}, at::kFloat, device, "t: fp32 [rows, rank] with unit column stride on the adapters' device", &t)) ||
      !workspace_of(a[11], need, device, &space, &have))
    return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_adapters(&w, x->data_ptr(), x_type, row_stride(*x), &rows, base ? base->data_ptr() : nullptr, base ? row_stride(*base) : 0, y.data_ptr(),
                        y_type, row_stride(y), has_t ? static_cast<float*>(t.data_ptr()) : nullptr, has_t ? row_stride(t) : 0,
                        have ? space.data_ptr() : nullptr, have, word, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return pack({returned(stream, a[7], y), has_t ? returned(stream, want_t, t) : Py_NewRef(Py_None)});
  END_HANDLE_TH_ERRORS
}

// (dy, x or None, a, b, t or None, order, groups, offsets, base, scale, dx, da, db (each None: not wanted, True: a new one), grad dtype or None,
//  workspace, status_word, stream) -> (dx, da, db), None where not wanted, or a status
PyObject* adapters_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!count_args(n, 17)) return nullptr;
  lcd_adapter_weights w = {};
  int32_t* word;
  at::Device device(at::kCPU);
  int64_t groups;
  lcd_row_groups rows;
  lcd_dtype type, other, grad_type = LCD_DTYPE_F32;
  if (!adapters_of(a[2], a[3], a[9], &w, &device) || !plan_of(a + 5, device, &groups, &rows) || !status_word_of(a[15], device, &word) ||
      !require(groups == w.G, "rows: a plan of as many groups as there are adapters"))
    return nullptr;
  const at::Tensor *dy = tensor_of(a[0], "dy"), *x = nullptr, *t = nullptr, *base = nullptr;
  if (!rows_of_x(dy, device, rows.count, w.N, &type, "dy: fp32, fp16 or bf16 [rows, N] with unit column stride on the adapters' device")) return nullptr;
  if (a[1] != Py_None) {
    x = tensor_of(a[1], "x");
    if (!rows_of_x(x, device, rows.count, w.K, &other, "x: [rows, K] of dy's type, with unit column stride, on the adapters' device") ||
        !require(other == type, "x: dy's type"))
      return nullptr;
  }
  if (a[4] != Py_None) {
    t = tensor_of(a[4], "t");
    if (!rows_of_x(t, device, rows.count, w.rank, &other, "t: fp32 [rows, rank] with unit column stride on the adapters' device") ||
        !require(other == LCD_DTYPE_F32, "t: fp32"))
      return nullptr;
  }
  if (a[8] != Py_None) {
    base = tensor_of(a[8], "base");
    if (!rows_of_x(base, device, rows.count, w.K, &other, "base: [rows, K] of dy's type, with unit column stride, on the adapters' device") ||
        !require(other == type, "base: dy's type"))
      return nullptr;
  }
  PyObject* want[3];
  bool has[3];
  for (int i = 0; i < 3; ++i) {
    has[i] = a[10 + i] != Py_None;
    want[i] = a[10 + i] == Py_True ? Py_None : a[10 + i];
  }
  at::ScalarType kind = tensor_of(a[2], "a")->scalar_type();
  if (a[13] != Py_None && !dtype_of(a[13], &kind)) return nullptr;
  if (a[13] == Py_None)
    for (int i = 1; i < 3; ++i)
      if (has[i] && want[i] != Py_None) {
        const at::Tensor* given = tensor_of(want[i], "da, db");
        if (!given) return nullptr;
        kind = given->scalar_type();
        break;
      }
  if (!require(type_of(kind, &grad_type), "da, db: fp32, fp16 or bf16") || !require(x || !has[1], "da: needs x") || !require(t || !has[2], "db: needs t")) return nullptr;
  const c10::cuda::CUDAGuard on(device);
  const CallStream stream(a[16]);
  if (!stream.ok()) return nullptr;
  size_t need = 0, have = 0;
  const lcd_status sized = lcd_adapters_workspace_bytes(rows.count, w.rank, &need);
  if (sized != LCD_OK) return PyLong_FromLong((long)sized);
  at::Tensor dx, da, db, space;
  if ((has[0] && !output_of(want[0], "dx", {rows.count, w.K}, dy->scalar_type(), device, "dx: [rows, K] of dy's type, with unit column stride, on the adapters' device", &dx)) ||
      (has[1] && (!output_of(want[1], "da", {w.G, w.rank, w.K}, kind, device, "da: [G, rank, K] on the adapters' device", &da) ||
                  !require(da.is_contiguous(), "da: contiguous"))) ||
      (has[2] && (!output_of(want[2], "db", {w.G, w.N, w.rank}, kind, device, "db: [G, N, rank] of da's type on the adapters' device", &db) ||
                  !require(db.is_contiguous(), "db: contiguous"))) ||
      !workspace_of(a[14], need, device, &space, &have))
    return nullptr;
  const lcd_status st = without_gil([&] {
    return lcd_adapters_grad(&w, dy->data_ptr(), row_stride(*dy), x ? x->data_ptr() : nullptr, x ? row_stride(*x) : 0, type,
                             t ? static_cast<const float*>(t->data_ptr()) : nullptr, t ? row_stride(*t) : 0, &rows, base ? base->data_ptr() : nullptr,
                             base ? row_stride(*base) : 0, has[0] ? dx.data_ptr() : nullptr, has[0] ? row_stride(dx) : 0,
                             has[1] ? da.data_ptr() : nullptr, has[2] ? db.data_ptr() : nullptr, grad_type, have ? space.data_ptr() : nullptr, have,
                             word, stream.raw());
  });
  if (st != LCD_OK) return PyLong_FromLong((long)st);
  return pack({has[0] ? returned(stream, want[0], dx) : Py_NewRef(Py_None), has[1] ? returned(stream, want[1], da) : Py_NewRef(Py_None),
               has[2] ? returned(stream, want[2], db) : Py_NewRef(Py_None)});
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
    {"smooth_quantize_act", reinterpret_cast<PyCFunction>(smooth_quantize_act), METH_FASTCALL, nullptr},
    {"lut_linear", reinterpret_cast<PyCFunction>(lut_linear), METH_FASTCALL, nullptr},
    {"act_batch", reinterpret_cast<PyCFunction>(act_batch), METH_FASTCALL, nullptr},
    {"linear_batch", reinterpret_cast<PyCFunction>(linear_batch), METH_FASTCALL, nullptr},
    {"reclassify", reinterpret_cast<PyCFunction>(reclassify), METH_FASTCALL, nullptr},
    {"smoothing_search", reinterpret_cast<PyCFunction>(smoothing_search), METH_FASTCALL, nullptr},
    {"mx_quantize", reinterpret_cast<PyCFunction>(mx_quantize), METH_FASTCALL, nullptr},
    {"mx_dequantize", reinterpret_cast<PyCFunction>(mx_dequantize), METH_FASTCALL, nullptr},
    {"mx_linear", reinterpret_cast<PyCFunction>(mx_linear), METH_FASTCALL, nullptr},
    {"distill", reinterpret_cast<PyCFunction>(distill), METH_FASTCALL, nullptr},
    {"group_rows", reinterpret_cast<PyCFunction>(group_rows), METH_FASTCALL, nullptr},
    {"mx_linear_grouped", reinterpret_cast<PyCFunction>(mx_linear_grouped), METH_FASTCALL, nullptr},
    {"adapters", reinterpret_cast<PyCFunction>(adapters), METH_FASTCALL, nullptr},
    {"adapters_grad", reinterpret_cast<PyCFunction>(adapters_grad), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls() { return PyModule_Create(&kModule); }
