// Argument marshalling of the serving calls for tensors of PyTorch, in C++: what binding.py does with ctypes for the prefill calls.
// A decode step issues a handful of calls whose kernels take a few microseconds each.  Through ctypes a call took 24 to 30 of the
// CPU's, here 4.8 to 8, of which a launch is 2.4 and decode attention makes two.  Checks, allocation of outputs, the current stream of
// the tensors' device; no arithmetic.
// The library's functions are handed over by address, so that the release and the debug library are bound alike.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "rbs.h"

namespace {

PyObject* error_class = nullptr;
PyObject* memory_class = nullptr;

decltype(&rbs_paged_extend) lib_extend = nullptr;
decltype(&rbs_qk_norm_rope) lib_norm_rope = nullptr;
decltype(&rbs_qk_norm_rope_paged) lib_norm_rope_paged = nullptr;
decltype(&rbs_paged_decode_workspace_bytes) lib_decode_workspace = nullptr;
decltype(&rbs_paged_decode) lib_decode = nullptr;
decltype(&rbs_status_string) lib_status_string = nullptr;

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};

std::string text(at::IntArrayRef sizes) {
  std::string s = "[";
  for (size_t i = 0; i < sizes.size(); ++i) s += (i ? ", " : "") + std::to_string(sizes[i]);
  return s + "]";
}

// The arguments of one call, whose tensors must all be on one CUDA device.
class Call {
 public:
  Call(const char* what, PyObject* const* args, Py_ssize_t have, Py_ssize_t want) : what_(what), args_(args) {
    if (lib_decode == nullptr) refuse("the library is not loaded");
    if (have != want) refuse("wrong number of arguments");
  }
  [[noreturn]] void refuse(const std::string& why) const { throw Refused(std::string(what_) + ": " + why); }

  bool given(int i) const { return args_[i] != Py_None; }
  const at::Tensor& tensor(int i) {
    if (!THPVariable_Check(args_[i])) refuse("expected a tensor");
    return on_device(THPVariable_Unpack(args_[i]));
  }
  const at::Tensor& on_device(const at::Tensor& t) {
    if (!t.is_cuda()) refuse("expected CUDA tensors");
    if (device_ < 0) device_ = t.get_device();
    if (t.get_device() != device_) refuse("tensors on cuda:" + std::to_string(device_) + " and cuda:" + std::to_string(t.get_device()));
    return t;
  }
  int integer(int i) const {
    const long long v = PyLong_AsLongLong(args_[i]);
    if (v == -1 && PyErr_Occurred()) throw std::exception();
    if (v < -0x80000000ll || v > 0x7fffffffll) refuse("a size is outside 32 bits");
    return static_cast<int>(v);
  }
  float number(int i) const {
    const double v = PyFloat_AsDouble(args_[i]);
    if (v == -1.0 && PyErr_Occurred()) throw std::exception();
    return static_cast<float>(v);
  }
  bool truth(int i) const {
    const int v = PyObject_IsTrue(args_[i]);
    if (v < 0) throw std::exception();
    return v != 0;
  }

  // a bf16 tensor of the given shape, [rows, heads, d] or [batch, rows, heads, d]; the stride of a dimension of one entry says nothing
  rbs_tensor rows(const at::Tensor& t, at::IntArrayRef shape) const {
    if (t.scalar_type() != at::kBFloat16 || t.dim() != static_cast<int64_t>(shape.size()) || t.stride(-1) != 1)
      refuse("expected a bf16 tensor " + text(shape) + " with the last dimension contiguous");
    if (t.sizes() != shape) refuse("expected shape " + text(shape) + ", got " + text(t.sizes()));
    const int64_t n = t.dim(), d = shape.back();
    auto stride = [&](int64_t k) { return shape[k] > 1 ? t.stride(k) : d; };
    return {t.data_ptr(), n == 4 ? stride(0) : 0, stride(n - 3), stride(n - 2)};
  }
  template <typename T>
  T* vector(const at::Tensor& t, int64_t n) const {
    const auto type = std::is_same<T, int>::value ? at::kInt : at::kFloat;
    if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
      refuse("expected " + std::to_string(n) + " contiguous " + (type == at::kInt ? "int32" : "fp32") + " values, got " + text(t.sizes()) +
             " of " + at::toString(t.scalar_type()));
    return static_cast<T*>(t.data_ptr());
  }
  // block table [sequences, pages] with contiguous rows
  void table(const at::Tensor& t, rbs_paged_shape& shape) const {
    if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) == 0 || t.size(1) == 0 || (t.size(1) > 1 && t.stride(1) != 1))
      refuse("expected an int32 block table [sequences, pages] with contiguous rows");
    shape.n_seqs = small(t.size(0));
    shape.max_pages = small(t.size(1));
    shape.table_stride = t.size(0) > 1 ? small(t.stride(0)) : shape.max_pages;
  }
  // the pair of caches [pages, page_size, kv_heads, d]
  void caches(const at::Tensor& k, const at::Tensor& v, int64_t d, rbs_paged_shape& shape, rbs_tensor& kt, rbs_tensor& vt) const {
    if (k.dim() != 4 || k.sizes() != v.sizes()) refuse("k_cache and v_cache must be [pages, page_size, kv_heads, " + std::to_string(d) + "]");
    const int64_t dims[4] = {k.size(0), k.size(1), k.size(2), d};
    kt = rows(k, dims);
    vt = rows(v, dims);
    shape.n_pages = small(dims[0]);
    shape.page_size = small(dims[1]);
    shape.n_kv_heads = small(dims[2]);
    shape.head_dim = small(d);
  }
  // positions, inv_freq, q_norm, k_norm, eps, interleaved, magnitude from argument i on
  rbs_rope rope(int i, int64_t tokens, int64_t d) {
    rbs_rope r = {};
    r.positions = vector<int>(tensor(i), tokens);
    if (given(i + 1)) {
      const at::Tensor& f = tensor(i + 1);
      if (f.numel() > 0) r.inv_freq = vector<float>(f, f.numel());
      r.rot_dim = small(2 * f.numel());
    }
    if (given(i + 2)) r.q_norm = vector<float>(tensor(i + 2), d);
    if (given(i + 3)) r.k_norm = vector<float>(tensor(i + 3), d);
    r.eps = number(i + 4);
    r.interleaved = truth(i + 5) ? 1 : 0;
    r.magnitude = number(i + 6);
    return r;
  }
  at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type) const {
    return at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, static_cast<c10::DeviceIndex>(device_)), std::nullopt);
  }
  at::Tensor output(int i, const at::Tensor& like) { return given(i) ? tensor(i) : fresh(like.sizes(), like.scalar_type()); }

  int small(int64_t v) const {
    if (v < -0x80000000ll || v > 0x7fffffffll) refuse("a size is outside 32 bits");
    return static_cast<int>(v);
  }
  int device() const { return device_; }
  // The library call, on the tensors' device and its current stream.
  template <typename F>
  void run(F&& f) const {
    const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(device_));
    const rbs_status st = f(static_cast<void*>(c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device_)).stream()));
    if (st != RBS_OK) throw Refused(std::string(what_) + " failed: " + lib_status_string(st));
  }

 private:
  const char* what_;
  PyObject* const* args_;
  int device_ = -1;
};

// No exception leaves a function that Python calls.
template <typename F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused& e) {
    PyErr_SetString(error_class, e.what());
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(memory_class, e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// n elements of a fresh 1-d tensor, from element `at` on, without the dispatcher
at::Tensor part_of(const at::Tensor& whole, int64_t at, int64_t n) {
  static const int64_t kOne = 1;
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
  t.unsafeGetTensorImpl()->set_sizes_and_strides(c10::IntArrayRef(&n, 1), c10::IntArrayRef(&kOne, 1), at);
  return t;
}

PyObject* pack(std::initializer_list<at::Tensor> ts) {
  PyObject* out = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
  if (out == nullptr) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = THPVariable_Wrap(t);
    if (o == nullptr) {
      Py_DECREF(out);
      return nullptr;
    }
    PyTuple_SET_ITEM(out, i++, o);
  }
  return out;
}

// seq_lens, new_lens, block_table, free_pages, page_size, n_pages, n_tokens, free_used, lens, cu, positions, slots, used
PyObject* extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c("rbs_paged_extend", args, n, 13);
    const at::Tensor &seq_lens = c.tensor(0), &new_lens = c.tensor(1), &table = c.tensor(2), &free = c.tensor(3);
    rbs_paged_shape shape = {};
    c.table(table, shape);
    shape.n_q_heads = shape.n_kv_heads = 1;
    shape.head_dim = 128;
    shape.page_size = c.integer(4);
    shape.n_pages = c.integer(5);
    const int tokens = c.integer(6);
    if (tokens < 0) c.refuse("n_tokens is negative");
    const int64_t sizes[5] = {shape.n_seqs, shape.n_seqs + 1ll, tokens, tokens, 1};
    at::Tensor out[5], all;
    int* p[5];
    if (!c.given(8)) {      // one allocation, 16-byte aligned parts
      int64_t n = 0;
      for (int64_t size : sizes) n += (size + 3) / 4 * 4;
      all = c.fresh({n}, at::kInt);
    }
    for (int64_t i = 0, at = 0; i < 5; at += (sizes[i] + 3) / 4 * 4, ++i) {
      out[i] = all.defined() ? part_of(all, at, sizes[i]) : c.tensor(static_cast<int>(8 + i));
      p[i] = c.vector<int>(out[i], sizes[i]);
    }
    const int *lens = c.vector<int>(seq_lens, shape.n_seqs), *more = c.vector<int>(new_lens, shape.n_seqs);
    const int* pages = c.vector<int>(free, free.numel());
    const int* used = c.given(7) ? c.vector<int>(c.tensor(7), 1) : nullptr;
    c.run([&](void* stream) {
      return lib_extend(&shape, lens, more, pages, c.small(free.numel()), used, tokens, static_cast<int*>(table.data_ptr()), p[0], p[1], p[2],
                        p[3], p[4], stream);
    });
    return pack({out[0], out[1], out[2], out[3], out[4]});
  });
}

// Q, K, positions, inv_freq, q_norm, k_norm, eps, interleaved, magnitude, out_q, out_k
PyObject* norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c("rbs_qk_norm_rope", args, n, 11);
    const at::Tensor &q = c.tensor(0), &k = c.tensor(1);
    const int64_t dims = q.dim();
    if ((dims != 3 && dims != 4) || k.dim() != dims || q.size(0) != k.size(0) || q.size(dims - 3) != k.size(dims - 3) || q.size(-1) != k.size(-1))
      c.refuse("Q and K must be [tokens, heads, 128] or [batch, tokens, heads, 128] with the same tokens");
    const int64_t tokens = q.size(dims - 3), d = q.size(-1);
    const rbs_rope rope = c.rope(2, tokens, d);
    const at::Tensor out_q = c.output(9, q), out_k = c.output(10, k);
    const rbs_tensor tq = c.rows(q, q.sizes()), tk = c.rows(k, k.sizes()), oq = c.rows(out_q, q.sizes()), ok = c.rows(out_k, k.sizes());
    c.run([&](void* stream) {
      return lib_norm_rope(dims == 4 ? c.small(q.size(0)) : 1, c.small(tokens), c.small(q.size(-2)), c.small(k.size(-2)), c.small(d), tq, tk, &rope,
                           oq, ok, stream);
    });
    return pack({out_q, out_k});
  });
}

// Q, K, V, positions, inv_freq, q_norm, k_norm, eps, interleaved, magnitude, slots, k_cache, v_cache, out_q, out_k
PyObject* norm_rope_paged(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c("rbs_qk_norm_rope_paged", args, n, 15);
    const at::Tensor &q = c.tensor(0), &k = c.tensor(1), &v = c.tensor(2), &slots = c.tensor(10), &kc = c.tensor(11), &vc = c.tensor(12);
    if (q.dim() != 3) c.refuse("Q must be [tokens, heads, 128]");
    const int64_t tokens = q.size(0), d = q.size(2);
    rbs_paged_shape shape = {};
    rbs_tensor tkc, tvc;
    c.caches(kc, vc, d, shape, tkc, tvc);
    shape.n_seqs = shape.max_pages = shape.table_stride = 1;
    shape.n_q_heads = c.small(q.size(1));
    const int64_t kv[3] = {tokens, shape.n_kv_heads, d};
    const rbs_rope rope = c.rope(3, tokens, d);
    if (slots.numel() > tokens) c.refuse("more slots than tokens");
    const at::Tensor out_q = c.output(13, q);
    const rbs_tensor tq = c.rows(q, q.sizes()), tk = c.rows(k, kv), tv = c.rows(v, kv), oq = c.rows(out_q, q.sizes());
    const rbs_tensor ok = c.given(14) ? c.rows(c.tensor(14), kv) : rbs_tensor{nullptr, 0, 0, 0};
    const int* s = c.vector<int>(slots, slots.numel());
    c.run([&](void* stream) {
      return lib_norm_rope_paged(&shape, c.small(tokens), tq, tk, tv, &rope, s, c.small(slots.numel()), oq, ok, tkc, tvc, stream);
    });
    return THPVariable_Wrap(out_q);
  });
}

// Q, k_cache, v_cache, block_table, seq_lens, out, return_lse, softmax_scale, workspace
PyObject* decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    Call c("rbs_paged_decode", args, n, 9);
    const at::Tensor &q = c.tensor(0), &kc = c.tensor(1), &vc = c.tensor(2), &table = c.tensor(3), &lens = c.tensor(4);
    if (q.dim() != 3) c.refuse("Q must be [sequences, heads, 128]");
    rbs_paged_shape shape = {};
    rbs_tensor tk, tv;
    c.caches(kc, vc, q.size(2), shape, tk, tv);
    c.table(table, shape);
    shape.n_q_heads = c.small(q.size(1));
    if (shape.n_seqs != q.size(0)) c.refuse(std::to_string(q.size(0)) + " rows of Q and " + std::to_string(shape.n_seqs) + " of the block table");
    const at::Tensor out = c.output(5, q);
    const rbs_tensor tq = c.rows(q, q.sizes()), to = c.rows(out, q.sizes());
    const int* l = c.vector<int>(lens, shape.n_seqs);
    at::Tensor lse, ws;
    if (c.truth(6)) lse = c.fresh({q.size(0), q.size(1)}, at::kFloat);
    const float scale = c.number(7);
    if (c.given(8)) {
      ws = c.tensor(8);
      if (ws.scalar_type() != at::kByte || !ws.is_contiguous()) c.refuse("the workspace must be a contiguous uint8 tensor");
    } else {
      ws = c.fresh({static_cast<int64_t>(lib_decode_workspace(&shape))}, at::kByte);
    }
    c.run([&](void* stream) {
      return lib_decode(&shape, tq, tk, tv, static_cast<const int*>(table.data_ptr()), l, to,
                        lse.defined() ? static_cast<float*>(lse.data_ptr()) : nullptr, scale, ws.data_ptr(), static_cast<size_t>(ws.numel()), stream);
    });
    return lse.defined() ? pack({out, lse}) : THPVariable_Wrap(out);
  });
}

// the error classes of refusals and of a full device, then the addresses of the library's functions
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 8) {
    PyErr_SetString(PyExc_TypeError, "bind: eight arguments");
    return nullptr;
  }
  void* at[6];
  for (int i = 0; i < 6; ++i) {
    at[i] = PyLong_AsVoidPtr(args[2 + i]);
    if (at[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: null address");
      return nullptr;
    }
  }
  Py_INCREF(args[0]);
  Py_INCREF(args[1]);
  Py_XDECREF(error_class);
  Py_XDECREF(memory_class);
  error_class = args[0];
  memory_class = args[1];
  lib_extend = reinterpret_cast<decltype(lib_extend)>(at[0]);
  lib_norm_rope = reinterpret_cast<decltype(lib_norm_rope)>(at[1]);
  lib_norm_rope_paged = reinterpret_cast<decltype(lib_norm_rope_paged)>(at[2]);
  lib_decode_workspace = reinterpret_cast<decltype(lib_decode_workspace)>(at[3]);
  lib_decode = reinterpret_cast<decltype(lib_decode)>(at[4]);
  lib_status_string = reinterpret_cast<decltype(lib_status_string)>(at[5]);
  Py_RETURN_NONE;
}

template <typename F>
PyCFunction method(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}

PyMethodDef methods[] = {{"bind", method(bind), METH_FASTCALL, nullptr},
                         {"paged_extend", method(extend), METH_FASTCALL, nullptr},
                         {"qk_norm_rope", method(norm_rope), METH_FASTCALL, nullptr},
                         {"qk_norm_rope_paged", method(norm_rope_paged), METH_FASTCALL, nullptr},
                         {"paged_decode", method(decode), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Marshalling of the serving calls; see binding.py.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
