// The product and conversion calls of the Python binding, and those around the key/value cache, as native functions: what they do between the caller and the C ABI
// (an output tensor, its address, the current stream) takes 2.4 us of a 5.8 us call in Python, and a small product is over
// on the GPU in 3.4.  Only plain device tensors and the current stream are served; for anything else the functions return None and
// the caller goes the general way through ctypes.  They call the entry points of the libmacko.so that is loaded already
// (bind() is given their addresses), and release the interpreter's lock around allocation and call, as ctypes does.
//
// Per call, through ctypes and here: a 512 x 512 product 5.8 and 4.9 us, a small batch product 7.8 and 5.6, a small decode 7.2 and
// 5.1.  Of the 4.9: 3.2 the runtime's launch (of an empty kernel as well), 0.2 the rest of the library, 0.3 the function
// here, 0.9 to 1.0 the output tensor (none if the caller gives one), 0.2 Python.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <pthread.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "macko.h"

namespace {

decltype(&macko_spmv) g_spmv = nullptr;
decltype(&macko_spmm) g_spmm = nullptr;
decltype(&macko_decode_device) g_decode = nullptr;
decltype(&macko_rotate) g_rotate = nullptr;
decltype(&macko_kv_append) g_append = nullptr;
decltype(&macko_kv_read) g_read = nullptr;
decltype(&macko_kv_attention_workspace) g_workspace = nullptr;
decltype(&macko_kv_attention) g_attention = nullptr;

// A forked child may not use its parent's device.  PyTorch's Python calls refuse that with an error, the C++ calls below do not:
// in a child the functions serve nothing, and the general way says what there is to say.
bool g_forked = false;

// A plain tensor on the GPU (no subclass: those may define what their methods do).
const at::Tensor* device_tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}

// What a call returns: its status as a number if it failed, else the tensor.
PyObject* result(int status, const at::Tensor& made, PyObject* given) {
  if (status != MACKO_OK) return PyLong_FromLong(status);
  if (given != Py_None) return Py_NewRef(given);
  return THPVariable_Wrap(made);
}

bool handle_of(PyObject* o, macko_handle_t* h) {       // None: a handle that has been destroyed
  *h = o == Py_None ? nullptr : static_cast<macko_handle_t>(PyLong_AsVoidPtr(o));
  return !PyErr_Occurred();
}

// spmv(handle, rows, x, y or None)
PyObject* spmv(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments");
  const at::Tensor* x = device_tensor(args[2]);
  const at::Tensor* given = args[3] == Py_None ? nullptr : device_tensor(args[3]);
  if (!g_spmv || g_forked || !x || (args[3] != Py_None && !given)) Py_RETURN_NONE;
  macko_handle_t h;
  if (!handle_of(args[0], &h)) return nullptr;
  const int64_t rows = PyLong_AsLongLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  at::Tensor y;
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    if (!given) y = at::empty({rows}, at::TensorOptions().dtype(at::kHalf).device(x->device()));
    status = g_spmv(h, x->data_ptr(), (given ? *given : y).data_ptr(), c10::hip::getCurrentHIPStream().stream());
  }
  return result(status, y, args[3]);
  END_HANDLE_TH_ERRORS
}

// spmm(handle, rows, X, Y or None)
PyObject* spmm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments");
  const at::Tensor* x = device_tensor(args[2]);
  const at::Tensor* given = args[3] == Py_None ? nullptr : device_tensor(args[3]);
  if (!g_spmm || g_forked || !x || (args[3] != Py_None && !given)) Py_RETURN_NONE;
  if (x->dim() != 2 || x->stride(1) != 1 || x->size(0) > MACKO_MAX_BATCH || (given && given->dim() != 2)) Py_RETURN_NONE;
  macko_handle_t h;
  if (!handle_of(args[0], &h)) return nullptr;
  const int64_t rows = PyLong_AsLongLong(args[1]), batch = x->size(0);
  if (PyErr_Occurred()) return nullptr;
  at::Tensor made;
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    if (!given) made = at::empty({batch, rows}, at::TensorOptions().dtype(at::kHalf).device(x->device()));
    const at::Tensor& y = given ? *given : made;
    const int64_t ldx = batch > 1 ? x->stride(0) : std::max<int64_t>(x->size(1), 1);
    const int64_t ldy = batch > 1 ? y.stride(0) : std::max<int64_t>(y.size(1), 1);
    status = g_spmm(h, (int)batch, x->data_ptr(), ldx, y.data_ptr(), ldy, c10::hip::getCurrentHIPStream().stream());
  }
  return result(status, made, args[3]);
  END_HANDLE_TH_ERRORS
}

// decode_device(handle, rows, cols, bits per value): into a new tensor on the current device
PyObject* decode_device(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 4) return PyErr_Format(PyExc_TypeError, "4 arguments");
  if (!g_decode || g_forked) Py_RETURN_NONE;
  macko_handle_t h;
  if (!handle_of(args[0], &h)) return nullptr;
  const int64_t rows = PyLong_AsLongLong(args[1]), cols = PyLong_AsLongLong(args[2]), bits = PyLong_AsLongLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  at::Tensor dense;
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    dense = at::empty({rows, cols}, at::TensorOptions().dtype(bits == 8 ? at::kByte : at::kHalf).device(at::kCUDA));
    status = g_decode(h, dense.data_ptr(), rows > 1 ? dense.stride(0) : std::max<int64_t>(cols, 1), c10::hip::getCurrentHIPStream().stream());
  }
  return result(status, dense, Py_None);
  END_HANDLE_TH_ERRORS
}

// ---- the key/value cache: kv.py makes the same checks and says what is wrong, so anything out of the ordinary is left to it ----

// A tensor argument that may be missing.
struct Given {
  const at::Tensor* t = nullptr;
  bool fine = true;
  explicit Given(PyObject* o) {
    if (o == Py_None) return;
    t = device_tensor(o);
    fine = t != nullptr;
  }
};

bool on(const at::Tensor& t, c10::DeviceIndex device) { return t.is_cuda() && t.get_device() == device; }

// [tokens, heads, dim] of 16 bits, channels next to each other
bool heads_fit(const at::Tensor& t, int64_t tokens, int64_t heads, int64_t dim, at::ScalarType type, c10::DeviceIndex device) {
  return t.dim() == 3 && t.size(0) == tokens && t.size(1) == heads && t.size(2) == dim && t.stride(2) == 1 && t.scalar_type() == type && on(t, device);
}
// the same for one that is written: whole rows one after the other
bool made_fits(const at::Tensor& t, int64_t tokens, int64_t heads, int64_t dim, at::ScalarType type, c10::DeviceIndex device) {
  return heads_fit(t, tokens, heads, dim, type, device) && t.stride(1) >= dim && t.stride(0) >= (heads - 1) * t.stride(1) + dim;
}
bool ints_fit(const at::Tensor& t, int64_t n, c10::DeviceIndex device) {
  return t.dim() == 1 && t.size(0) == n && t.stride(0) == 1 && t.scalar_type() == at::kInt && on(t, device);
}
bool weight_fits(const Given& w, int64_t dim, at::ScalarType type, c10::DeviceIndex device) {
  return w.fine && (!w.t || (w.t->dim() == 1 && w.t->size(0) == dim && w.t->stride(0) == 1 && w.t->scalar_type() == type && on(*w.t, device)));
}
bool rotation_of(const Given& positions, const Given& table, int64_t tokens, int interleaved, double eps, c10::DeviceIndex device, macko_rotation_t* r) {
  *r = macko_rotation_t{nullptr, nullptr, 0, 0, 0, (float)eps};
  if (!positions.fine || !table.fine) return false;
  if (!table.t) return true;
  const at::Tensor& t = *table.t;
  if (!positions.t || !ints_fit(*positions.t, tokens, device) || t.dim() != 3 || t.size(1) != 2 || t.size(2) > 128 || t.scalar_type() != at::kFloat || !t.is_contiguous() || !on(t, device))
    return false;
  *r = macko_rotation_t{static_cast<const int32_t*>(positions.t->data_ptr()), static_cast<const float*>(t.data_ptr()), t.size(0), (int32_t)(2 * t.size(2)), interleaved, (float)eps};
  return true;
}
int type_of(const at::Tensor& t) { return t.scalar_type() == at::kHalf ? MACKO_FP16 : t.scalar_type() == at::kBFloat16 ? MACKO_BF16 : -1; }
at::Tensor made_heads(int64_t tokens, int64_t heads, int64_t dim, const at::Tensor& like) { return at::empty({tokens, heads, dim}, like.options()); }

// rotate(x, positions, table, weight, eps, interleaved, out)
PyObject* rotate(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments");
  const Given x(args[0]), positions(args[1]), table(args[2]), weight(args[3]), out(args[6]);
  const double eps = PyFloat_AsDouble(args[4]);
  const int interleaved = PyObject_IsTrue(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!g_rotate || g_forked || !x.t || x.t->dim() != 3 || !out.fine) Py_RETURN_NONE;
  const c10::DeviceIndex device = c10::hip::current_device();
  const int64_t tokens = x.t->size(0), heads = x.t->size(1), dim = x.t->size(2);
  const int type = type_of(*x.t);
  macko_rotation_t r;
  if (type < 0 || !heads_fit(*x.t, tokens, heads, dim, x.t->scalar_type(), device) || !weight_fits(weight, dim, x.t->scalar_type(), device) ||
      !rotation_of(positions, table, tokens, interleaved, eps, device, &r) || (out.t && !made_fits(*out.t, tokens, heads, dim, x.t->scalar_type(), device)) ||
      heads > INT32_MAX || dim > INT32_MAX)
    Py_RETURN_NONE;
  at::Tensor made;
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    if (!out.t) made = made_heads(tokens, heads, dim, *x.t);
    const at::Tensor& y = out.t ? *out.t : made;
    status = g_rotate(tokens, (int)heads, (int)dim, type, x.t->data_ptr(), x.t->stride(0), x.t->stride(1), &r, weight.t ? weight.t->data_ptr() : nullptr,
                      y.data_ptr(), y.stride(0), y.stride(1), c10::hip::getCurrentHIPStream().stream());
  }
  return result(status, made, args[6]);
  END_HANDLE_TH_ERRORS
}

// The cache's geometry and its device, from their address and number.
const macko_kv_cache_t* cache_of(PyObject* address, PyObject* device, c10::DeviceIndex* current) {
  const auto* c = static_cast<const macko_kv_cache_t*>(PyLong_AsVoidPtr(address));
  const long d = PyLong_AsLong(device);
  *current = c10::hip::current_device();
  return d == *current ? c : nullptr;
}

// kv_append(cache, device, q, k, v, positions, slots, table, q_weight, k_weight, eps, interleaved, q_out): True without queries
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 13) return PyErr_Format(PyExc_TypeError, "13 arguments");
  c10::DeviceIndex device;
  const macko_kv_cache_t* cache = cache_of(args[0], args[1], &device);
  const Given q(args[2]), k(args[3]), v(args[4]), positions(args[5]), slots(args[6]), table(args[7]), q_weight(args[8]), k_weight(args[9]), out(args[12]);
  const double eps = PyFloat_AsDouble(args[10]);
  const int interleaved = PyObject_IsTrue(args[11]);
  if (PyErr_Occurred()) return nullptr;
  if (!g_append || g_forked || !cache || !k.t || !v.t || !slots.t || k.t->dim() != 3 || !q.fine || !out.fine || (q.t && q.t->dim() != 3)) Py_RETURN_NONE;
  const at::ScalarType scalar = k.t->scalar_type();
  const int64_t tokens = k.t->size(0), heads = q.t ? q.t->size(1) : 0, dim = cache->head_dim;
  macko_kv_append_args_t a{};
  a.tokens = tokens;
  a.heads = (int32_t)heads;
  a.type = type_of(*k.t);
  if (a.type < 0 || heads > INT32_MAX || !heads_fit(*k.t, tokens, cache->kv_heads, dim, scalar, device) || !heads_fit(*v.t, tokens, cache->kv_heads, dim, scalar, device) ||
      !ints_fit(*slots.t, tokens, device) || (q.t && !heads_fit(*q.t, tokens, heads, dim, scalar, device)) || !weight_fits(k_weight, dim, scalar, device) ||
      !weight_fits(q_weight, dim, scalar, device) || !rotation_of(positions, table, tokens, interleaved, eps, device, &a.rotation) ||
      (q.t && out.t && !made_fits(*out.t, tokens, heads, dim, scalar, device)))
    Py_RETURN_NONE;
  a.k_dev = k.t->data_ptr(), a.k_token = k.t->stride(0), a.k_head = k.t->stride(1);
  a.v_dev = v.t->data_ptr(), a.v_token = v.t->stride(0), a.v_head = v.t->stride(1);
  a.slots_dev = static_cast<const int32_t*>(slots.t->data_ptr());
  a.k_weight_dev = k_weight.t ? k_weight.t->data_ptr() : nullptr;
  a.q_weight_dev = q.t && q_weight.t ? q_weight.t->data_ptr() : nullptr;
  at::Tensor made;
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    if (q.t) {
      if (!out.t) made = made_heads(tokens, heads, dim, *q.t);
      const at::Tensor& y = out.t ? *out.t : made;
      a.q_dev = q.t->data_ptr(), a.q_token = q.t->stride(0), a.q_head = q.t->stride(1);
      a.q_out_dev = y.data_ptr(), a.q_out_token = y.stride(0), a.q_out_head = y.stride(1);
    }
    status = g_append(cache, &a, c10::hip::getCurrentHIPStream().stream());
  }
  if (status == MACKO_OK && !q.t) Py_RETURN_TRUE;
  return result(status, made, args[12]);
  END_HANDLE_TH_ERRORS
}

// A pair of tensors, or the status of a call that failed.
PyObject* two(int status, const at::Tensor& a, PyObject* given_a, const at::Tensor& b, PyObject* given_b) {
  if (status != MACKO_OK) return PyLong_FromLong(status);
  PyObject* x = given_a != Py_None ? Py_NewRef(given_a) : THPVariable_Wrap(a);
  PyObject* y = x ? (given_b != Py_None ? Py_NewRef(given_b) : THPVariable_Wrap(b)) : nullptr;
  PyObject* pair = y ? PyTuple_New(2) : nullptr;
  if (!pair) {
    Py_XDECREF(x);
    Py_XDECREF(y);
    return nullptr;
  }
  PyTuple_SET_ITEM(pair, 0, x);
  PyTuple_SET_ITEM(pair, 1, y);
  return pair;
}

// kv_read(cache, device, slots, bf16, k_out, v_out)
PyObject* kv_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6) return PyErr_Format(PyExc_TypeError, "6 arguments");
  c10::DeviceIndex device;
  const macko_kv_cache_t* cache = cache_of(args[0], args[1], &device);
  const Given slots(args[2]), k(args[4]), v(args[5]);
  const bool bf16 = PyObject_IsTrue(args[3]);
  if (PyErr_Occurred()) return nullptr;
  if (!g_read || g_forked || !cache || !slots.t || slots.t->dim() != 1 || !k.fine || !v.fine) Py_RETURN_NONE;
  const at::ScalarType scalar = bf16 ? at::kBFloat16 : at::kHalf;
  const int64_t tokens = slots.t->size(0), heads = cache->kv_heads, dim = cache->head_dim;
  if (!ints_fit(*slots.t, tokens, device) || (k.t && !made_fits(*k.t, tokens, heads, dim, scalar, device)) || (v.t && !made_fits(*v.t, tokens, heads, dim, scalar, device)))
    Py_RETURN_NONE;
  at::Tensor made[2];
  int status;
  {
    pybind11::gil_scoped_release unlocked;
    const auto options = at::TensorOptions().dtype(scalar).device(slots.t->device());
    if (!k.t) made[0] = at::empty({tokens, heads, dim}, options);
    if (!v.t) made[1] = at::empty({tokens, heads, dim}, options);
    const at::Tensor &x = k.t ? *k.t : made[0], &y = v.t ? *v.t : made[1];
    status = g_read(cache, tokens, static_cast<const int32_t*>(slots.t->data_ptr()), bf16 ? MACKO_BF16 : MACKO_FP16, x.data_ptr(), x.stride(0), x.stride(1), y.data_ptr(),
                    y.stride(0), y.stride(1), c10::hip::getCurrentHIPStream().stream());
  }
  return two(status, made[0], args[4], made[1], args[5]);
  END_HANDLE_TH_ERRORS
}

// kv_attend(cache, device, q, tables, lengths, start, most_queries, longest or None, scale or None, window, sums, out)
PyObject* kv_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 12) return PyErr_Format(PyExc_TypeError, "12 arguments");
  c10::DeviceIndex device;
  const macko_kv_cache_t* cache = cache_of(args[0], args[1], &device);
  const Given q(args[2]), tables(args[3]), lengths(args[4]), start(args[5]), out(args[11]);
  const int64_t most = PyLong_AsLongLong(args[6]), window = PyLong_AsLongLong(args[9]), longest = args[7] == Py_None ? -1 : PyLong_AsLongLong(args[7]);
  const double scale = args[8] == Py_None ? 0.0 : PyFloat_AsDouble(args[8]);
  const bool sums = PyObject_IsTrue(args[10]);
  if (PyErr_Occurred()) return nullptr;
  if (!g_attention || g_forked || !cache || !q.t || !tables.t || !lengths.t || !start.fine || !out.fine || q.t->dim() != 3 || tables.t->dim() != 2 || lengths.t->dim() != 1)
    Py_RETURN_NONE;
  const int64_t tokens = q.t->size(0), heads = q.t->size(1), dim = cache->head_dim, batch = lengths.t->size(0), width = tables.t->size(1);
  const at::ScalarType scalar = q.t->scalar_type();
  macko_kv_attention_args_t a{};
  a.type = type_of(*q.t);
  if (a.type < 0 || tokens == 0 || heads > INT32_MAX || batch > INT32_MAX || width > INT32_MAX || most < 1 || most > INT32_MAX || window < 0 || window > INT32_MAX ||
      longest < (args[7] == Py_None ? -1 : 0) || !heads_fit(*q.t, tokens, heads, dim, scalar, device) || !ints_fit(*lengths.t, batch, device) || tables.t->size(0) != batch ||
      tables.t->scalar_type() != at::kInt || (width > 1 && tables.t->stride(1) != 1) || !on(*tables.t, device) || (start.t ? !ints_fit(*start.t, batch + 1, device) : batch != tokens) ||
      (out.t && !made_fits(*out.t, tokens, heads, dim, scalar, device)))
    Py_RETURN_NONE;
  a.tokens = tokens, a.heads = (int32_t)heads, a.batch = (int32_t)batch;
  a.q_dev = q.t->data_ptr(), a.q_token = q.t->stride(0), a.q_head = q.t->stride(1);
  a.tables_dev = static_cast<const int32_t*>(tables.t->data_ptr()), a.table_stride = tables.t->stride(0), a.table_width = (int32_t)width;
  a.lengths_dev = static_cast<const int32_t*>(lengths.t->data_ptr());
  a.start_dev = start.t ? static_cast<const int32_t*>(start.t->data_ptr()) : nullptr;
  a.most_queries = (int32_t)most, a.window = (int32_t)window;
  a.longest = longest < 0 ? width * cache->page_size : longest;
  a.scale = args[8] == Py_None ? (float)(1.0 / std::sqrt((double)dim)) : (float)scale;
  at::Tensor made, total;
  int64_t status;
  {
    pybind11::gil_scoped_release unlocked;
    status = g_workspace(cache, &a);
    if (status >= 0) {
      at::Tensor work;
      if (!out.t) made = made_heads(tokens, heads, dim, *q.t);
      const at::Tensor& y = out.t ? *out.t : made;
      a.out_dev = y.data_ptr(), a.out_token = y.stride(0), a.out_head = y.stride(1);
      if (sums) {
        total = at::empty({tokens, heads}, q.t->options().dtype(at::kFloat));
        a.sums_dev = static_cast<float*>(total.data_ptr());
      }
      if (status > 0) work = at::empty({status}, q.t->options().dtype(at::kByte));
      status = g_attention(cache, &a, status > 0 ? work.data_ptr() : nullptr, status, c10::hip::getCurrentHIPStream().stream());
    }
  }
  if (sums) return two((int)status, made, args[11], total, Py_None);
  return result((int)status, made, args[11]);
  END_HANDLE_TH_ERRORS
}

// bind(addresses of macko_spmv, macko_spmm, macko_decode_device, macko_rotate, macko_kv_append, macko_kv_read, macko_kv_attention_workspace,
// macko_kv_attention)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "8 arguments");
  void* p[8];
  for (int i = 0; i < 8; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  if (!g_spmv && pthread_atfork(nullptr, nullptr, [] { g_forked = true; }) != 0) return PyErr_NoMemory();
  g_spmv = reinterpret_cast<decltype(g_spmv)>(p[0]);
  g_spmm = reinterpret_cast<decltype(g_spmm)>(p[1]);
  g_decode = reinterpret_cast<decltype(g_decode)>(p[2]);
  g_rotate = reinterpret_cast<decltype(g_rotate)>(p[3]);
  g_append = reinterpret_cast<decltype(g_append)>(p[4]);
  g_read = reinterpret_cast<decltype(g_read)>(p[5]);
  g_workspace = reinterpret_cast<decltype(g_workspace)>(p[6]);
  g_attention = reinterpret_cast<decltype(g_attention)>(p[7]);
  Py_RETURN_NONE;
}

#define MACKO_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MACKO_FAST(spmv), MACKO_FAST(spmm), MACKO_FAST(decode_device), MACKO_FAST(rotate), MACKO_FAST(kv_append), MACKO_FAST(kv_read), MACKO_FAST(kv_attend), MACKO_FAST(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
