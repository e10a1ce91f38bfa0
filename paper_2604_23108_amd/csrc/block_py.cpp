// Marshalling of the calls of mohge_block.h for Python: shapes, types, strides and addresses of the tensors
// and the current stream, handed to the C entry points (whose addresses `bind` receives).  Extension module
// `_block_native` of the package.
//
// The calls of a decode step run for 2 to 10 us on the GPU; looked at through Python attributes and ctypes, the tensors of one
// call cost 5.7 (six tensors) to 10 us (twelve) of host time, which is then the limit.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include <initializer_list>
#include <string>

#include "mohge_block.h"

namespace {

struct Entry {
  decltype(&mohge_rmsnorm) rmsnorm;
  decltype(&mohge_rmsnorm_bwd) rmsnorm_bwd;
  decltype(&mohge_cache_append) cache_append;
  decltype(&mohge_cache_attention) cache_attention;
  decltype(&mohge_proj_w4) proj_w4;
  decltype(&mohge_last_error) last_error;
};
Entry g_entry;
PyObject* g_error;      // MohgeError

struct Refused {};       // a Python exception is set

[[noreturn]] void refuse(const std::string& text) {
  PyErr_SetString(g_error, text.c_str());
  throw Refused();
}

const char* type_name(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return "torch.bfloat16";
    case at::kFloat: return "torch.float32";
    case at::kByte: return "torch.uint8";
    case at::kInt: return "torch.int32";
    default: return c10::toString(t);
  }
}

std::string shape_name(c10::ArrayRef<int64_t> s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + (s.size() == 1 ? ",)" : ")");
}

// storage of the configurations' types
at::ScalarType torch_type(int dtype) {
  return dtype == MOHGE_BF16 ? at::kBFloat16 : dtype == MOHGE_F32 ? at::kFloat : at::kByte;
}

const at::Tensor& tensor_of(const char* name, PyObject* o) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is needed");
  return THPVariable_Unpack(o);
}

void expect(const char* name, const at::Tensor& t, c10::ArrayRef<int64_t> shape, at::ScalarType type) {
  if (t.sizes() != shape || t.scalar_type() != type)
    refuse(std::string(name) + ": " + shape_name(t.sizes()) + " " + type_name(t.scalar_type()) + " given, " + shape_name(shape) +
           " " + type_name(type) + " needed");
  if (!t.is_cuda()) refuse("tensors handed to the library must be on the GPU");
}

// address of a contiguous tensor of this shape and type; None stays NULL (the library says what it needs)
template <typename T = void>
T* at_of(const char* name, PyObject* o, std::initializer_list<int64_t> shape, at::ScalarType type) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor_of(name, o);
  expect(name, t, c10::ArrayRef<int64_t>(shape.begin(), shape.size()), type);
  if (!t.is_contiguous()) refuse("tensors handed to the library must be contiguous");
  return static_cast<T*>(t.data_ptr());
}

// [rows, heads, size] whose rows are contiguous but may be further apart
void* rows_of(const char* name, PyObject* o, int64_t rows, int64_t heads, int64_t size, at::ScalarType type, int64_t* stride) {
  const at::Tensor& t = tensor_of(name, o);
  expect(name, t, {rows, heads, size}, type);
  if (t.stride(2) != 1 || (t.stride(1) != size && heads > 1)) refuse(std::string(name) + ": the heads of a row must be contiguous");
  *stride = rows > 1 ? t.stride(0) : heads * size;
  return t.data_ptr();
}

void* bytes_of(const char* name, PyObject* o, size_t* bytes) {
  *bytes = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor_of(name, o);
  if (!t.is_cuda()) refuse("tensors handed to the library must be on the GPU");
  if (!t.is_contiguous()) refuse("tensors handed to the library must be contiguous");
  *bytes = t.nbytes();
  return t.data_ptr();
}

template <typename T>
const T& config_of(PyObject* o) {
  const void* p = PyLong_AsVoidPtr(o);
  if (!p) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "the address of a configuration is needed");
    throw Refused();
  }
  return *static_cast<const T*>(p);
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

void check(int rc, const char* what) {
  if (rc) refuse(std::string(what) + " failed with code " + std::to_string(rc) + ": " + g_entry.last_error());
}

// no C++ exception leaves a call
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "%zd arguments given, %zd needed", given, wanted);
    return nullptr;
  }
  try {
    f();
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown exception");
    return nullptr;
  }
  Py_RETURN_NONE;
}

PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const auto& c = config_of<mohge_norm_config>(a[0]);
    const at::ScalarType t = torch_type(c.dtype);
    const void* x = at_of("x", a[1], {c.T, c.d}, t);
    const void* residual = at_of("residual", a[2], {c.T, c.d}, t);
    const float* weight = at_of<float>("weight", a[3], {c.d}, at::kFloat);
    void* sum = at_of("sum_out", a[4], {c.T, c.d}, t);
    void* y = at_of("y", a[5], {c.T, c.d}, torch_type(c.y_dtype));
    float* y_scale = at_of<float>("y_scale", a[6], {c.T}, at::kFloat);
    float* rstd = at_of<float>("rstd", a[7], {c.T}, at::kFloat);
    check(g_entry.rmsnorm(&c, x, residual, weight, sum, y, y_scale, rstd, stream()), "mohge_rmsnorm");
  });
}

PyObject* rmsnorm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const auto& c = config_of<mohge_norm_config>(a[0]);
    const at::ScalarType t = torch_type(c.dtype);
    const void* dy = at_of("dy", a[1], {c.T, c.d}, t);
    const void* h = at_of("h", a[2], {c.T, c.d}, t);
    const float* weight = at_of<float>("weight", a[3], {c.d}, at::kFloat);
    const float* rstd = at_of<float>("rstd", a[4], {c.T}, at::kFloat);
    const void* dsum = at_of("dsum", a[5], {c.T, c.d}, t);
    void* dx = at_of("dx", a[6], {c.T, c.d}, t);
    float* dweight = at_of<float>("dweight", a[7], {c.d}, at::kFloat);
    size_t bytes;
    void* ws = bytes_of("workspace", a[8], &bytes);
    check(g_entry.rmsnorm_bwd(&c, dy, h, weight, rstd, dsum, dx, dweight, ws, bytes, stream()), "mohge_rmsnorm_bwd");
  });
}

// block_table, seq_lens, k_pages, v_pages, k_scale, v_scale
struct CacheTensors {
  const int32_t *table, *lens;
  void *k, *v;
  float *ks, *vs;
  CacheTensors(const mohge_cache_config& c, PyObject* const* a) {
    const at::ScalarType t = torch_type(c.cache_dtype);
    table = at_of<int32_t>("block_table", a[0], {c.n_seqs, c.max_pages}, at::kInt);
    lens = at_of<int32_t>("seq_lens", a[1], {c.n_seqs}, at::kInt);
    k = at_of("k_pages", a[2], {c.n_pages, c.n_kv_heads, c.page_size, c.head_size}, t);
    v = at_of("v_pages", a[3], {c.n_pages, c.n_kv_heads, c.page_size, c.head_size}, t);
    ks = at_of<float>("k_scale", a[4], {c.n_pages, c.n_kv_heads, c.page_size}, at::kFloat);
    vs = at_of<float>("v_scale", a[5], {c.n_pages, c.n_kv_heads, c.page_size}, at::kFloat);
  }
};

PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const auto& c = config_of<mohge_cache_config>(a[0]);
    const at::ScalarType t = torch_type(c.dtype);
    const at::Tensor& first = tensor_of("k", a[1]);
    if (first.dim() != 3) refuse("k: [rows, heads, size] needed");
    const int64_t rows = first.size(0);
    if (rows > INT32_MAX) refuse("k: fewer than 2^31 rows needed");
    int64_t k_stride, v_stride;
    const void* k = rows_of("k", a[1], rows, c.n_kv_heads, c.head_size, t, &k_stride);
    const void* v = rows_of("v", a[2], rows, c.n_kv_heads, c.head_size, t, &v_stride);
    const int32_t* offsets = at_of<int32_t>("tok_offsets", a[3], {(int64_t)c.n_seqs + 1}, at::kInt);
    const CacheTensors x(c, a + 4);
    check(g_entry.cache_append(&c, (int32_t)rows, k, k_stride, v, v_stride, offsets, x.table, x.lens, x.k, x.v, x.ks, x.vs, stream()),
          "mohge_cache_append");
  });
}

PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    const auto& c = config_of<mohge_cache_config>(a[0]);
    const at::ScalarType t = torch_type(c.dtype);
    int64_t q_stride;
    const void* q = rows_of("q", a[1], c.n_seqs, c.n_heads, c.head_size, t, &q_stride);
    const CacheTensors x(c, a + 2);
    const double scale = PyFloat_AsDouble(a[8]);
    if (PyErr_Occurred()) throw Refused();
    void* out = at_of("out", a[9], {c.n_seqs, c.n_heads, c.head_size}, t);
    float* lse = at_of<float>("lse", a[10], {c.n_seqs, c.n_heads}, at::kFloat);
    size_t bytes;
    void* ws = bytes_of("workspace", a[11], &bytes);
    check(g_entry.cache_attention(&c, q, q_stride, x.table, x.lens, x.k, x.v, x.ks, x.vs, (float)scale, out, lse, ws, bytes, stream()),
          "mohge_cache_attention");
  });
}

PyObject* proj_w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const auto& c = config_of<mohge_proj_config>(a[0]);
    const int64_t groups = c.group > 0 ? c.n_in / c.group : 0;
    const void* x = at_of("x", a[1], {c.T, c.n_in}, torch_type(c.x_dtype));
    const float* x_scale = at_of<float>("x_scale", a[2], {c.T}, at::kFloat);
    const void* codes = at_of("codes", a[3], {c.n_out, c.n_in / 2}, at::kByte);
    const void* scales = at_of("scales", a[4], {c.n_out, groups}, at::kBFloat16);
    const void* zeros = at_of("zeros", a[5], {c.n_out, groups}, at::kByte);
    void* y = at_of("y", a[6], {c.T, c.n_out}, torch_type(c.y_dtype));
    check(g_entry.proj_w4(&c, x, x_scale, codes, scales, zeros, y, stream()), "mohge_proj_w4");
  });
}

// bind(error class, addresses of the entry points in the order of Entry)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    void* p[6];
    for (int i = 0; i < 6; ++i) {
      p[i] = PyLong_AsVoidPtr(a[i + 1]);
      if (!p[i]) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "the address of an entry point is needed");
        throw Refused();
      }
    }
    Py_INCREF(a[0]);
    Py_XDECREF(g_error);
    g_error = a[0];
    g_entry.rmsnorm = reinterpret_cast<decltype(g_entry.rmsnorm)>(p[0]);
    g_entry.rmsnorm_bwd = reinterpret_cast<decltype(g_entry.rmsnorm_bwd)>(p[1]);
    g_entry.cache_append = reinterpret_cast<decltype(g_entry.cache_append)>(p[2]);
    g_entry.cache_attention = reinterpret_cast<decltype(g_entry.cache_attention)>(p[3]);
    g_entry.proj_w4 = reinterpret_cast<decltype(g_entry.proj_w4)>(p[4]);
    g_entry.last_error = reinterpret_cast<decltype(g_entry.last_error)>(p[5]);
  });
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {METHOD(bind), METHOD(rmsnorm), METHOD(rmsnorm_bwd), METHOD(cache_append), METHOD(cache_attention),
                           METHOD(proj_w4), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_block_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block_native(void) { return PyModule_Create(&g_module); }
