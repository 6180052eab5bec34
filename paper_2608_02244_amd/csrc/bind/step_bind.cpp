// Python binding of the step's operators (module paper_2608_02244_amd._step): checks
// of torch tensors, outputs, and the C calls of fsched.h.  In C++ because a small
// decode step is a few microseconds of GPU work per call: the same marshalling in
// Python took 7 to 10 us a call.  step.py documents the calls and gives them keywords.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/MemoryOverlap.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <string>

#include "fsched.h"

namespace {

struct Refused {  // becomes a ValueError
  std::string what;
};
struct Raised {};  // a Python error is set

std::string dtype_name(at::ScalarType t) {
  return t == at::kBFloat16 ? "torch.bfloat16" : t == at::kHalf ? "torch.float16" : "other";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused{std::string(name) + " must be a tensor"};
  return THPVariable_Unpack(o);
}

// The tensors among a call's arguments lie on one device, which is current during the
// call (kernels read all of them, and the library launches on the current device).
c10::DeviceGuard one_device(PyObject* const* a, Py_ssize_t n) {
  const at::Tensor* first = nullptr;
  for (Py_ssize_t i = 0; i < n; ++i) {
    // numbers first: the tensor check is an isinstance() for them (0.2 us a call in all)
    if (a[i] == Py_None || PyLong_Check(a[i]) || PyFloat_Check(a[i])) continue;
    if (!THPVariable_Check(a[i])) continue;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (!first) first = &t;
    else if (t.device() != first->device())
      throw Refused{"all tensors of a call must be on one GPU"};
  }
  if (!first) throw Refused{"the first argument must be a GPU tensor"};
  return c10::DeviceGuard(first->device());
}

int64_t integer(PyObject* o, int64_t lo, int64_t hi, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < lo || v > hi) throw Refused{std::string(name) + " is out of range"};
  return v;
}
int32_t int32(PyObject* o, const char* name) {
  return (int32_t)integer(o, INT32_MIN, INT32_MAX, name);
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return (float)v;
}
void* handle(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

int32_t extent(int64_t n, const char* name) {
  if (n > INT32_MAX) throw Refused{std::string(name) + " is too long"};
  return (int32_t)n;
}

// A contiguous int32 GPU tensor of one dimension (n elements, any if n < 0).
int32_t* ints(PyObject* o, int64_t n, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kInt || !t.is_cuda() || t.dim() != 1 || !t.is_contiguous() ||
      (n >= 0 && t.size(0) != n))
    throw Refused{std::string(name) + " must be a contiguous int32 GPU tensor of shape (" +
                  (n < 0 ? std::string("any") : std::to_string(n)) + ",)"};
  return (int32_t*)t.data_ptr();
}

int32_t* table(PyObject* o, int64_t n, int32_t* width) {
  const at::Tensor& t = tensor(o, "block_table");
  if (t.scalar_type() != at::kInt || !t.is_cuda() || t.dim() != 2 || !t.is_contiguous() ||
      t.size(0) != n)
    throw Refused{"block_table must be a contiguous int32 GPU tensor of shape (" +
                  std::to_string(n) + ", any)"};
  *width = extent(t.size(1), "block_table");
  return (int32_t*)t.data_ptr();
}

// A GPU tensor of `dim` dimensions and the cache's type, the last one contiguous.
const at::Tensor& rows(PyObject* o, int64_t dim, at::ScalarType type, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != dim || t.scalar_type() != type || !t.is_cuda() ||
      (t.stride(dim - 1) != 1 && t.size(dim - 1) > 1))
    throw Refused{std::string(name) + " must be a " + std::to_string(dim) + "-dimensional " +
                  dtype_name(type) + " GPU tensor whose last dimension is contiguous"};
  return t;
}

// What a call writes: no two of its elements may be one.
void written(const at::Tensor& t, const char* name) {
  if (at::has_internal_overlap(t) == at::MemOverlap::Yes)
    throw Refused{std::string(name) + " is written and must not be an expanded tensor"};
}

struct Cache {
  fsched_kv_cache c;
  at::ScalarType type;
};

Cache cache(PyObject* ko, PyObject* vo) {
  const at::Tensor& k0 = tensor(ko, "k_cache");
  const at::ScalarType type = k0.scalar_type();
  if (type != at::kBFloat16 && type != at::kHalf)
    throw Refused{"the cache must be bfloat16 or float16"};
  const at::Tensor& k = rows(ko, 4, type, "k_cache");
  const at::Tensor& v = rows(vo, 4, type, "v_cache");
  if (k.sizes() != v.sizes()) throw Refused{"k_cache and v_cache differ in shape"};
  Cache r;
  r.type = type;
  r.c = fsched_kv_cache{};
  r.c.k = k.data_ptr();
  r.c.v = v.data_ptr();
  for (int i = 0; i < 3; ++i) {
    r.c.k_stride[i] = k.stride(i);
    r.c.v_stride[i] = v.stride(i);
  }
  r.c.n_pages = extent(k.size(0), "k_cache");
  r.c.kv_heads = extent(k.size(1), "k_cache");
  r.c.page_size = extent(k.size(2), "k_cache");
  r.c.head_dim = extent(k.size(3), "k_cache");
  r.c.dtype = type == at::kBFloat16 ? FSCHED_BF16 : FSCHED_F16;
  return r;
}

// A return code as the package's FschedError.
void check(int rc, const char* name) {
  if (rc == FSCHED_OK) return;
  PyObject* m = PyImport_ImportModule("paper_2608_02244_amd");
  PyObject* cls = m ? PyObject_GetAttrString(m, "FschedError") : nullptr;
  PyObject* e = cls ? PyObject_CallFunction(cls, "is", rc, name) : nullptr;
  if (e) PyErr_SetObject(cls, e);
  Py_XDECREF(e);
  Py_XDECREF(cls);
  Py_XDECREF(m);
  throw Raised{};
}

// Runs `body` and turns what it throws into Python errors.
template <class F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F body) {
  if (got != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Raised&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what.c_str());
  } catch (...) {  // torch's errors as torch raises them (torch.OutOfMemoryError, ...)
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

at::TensorOptions like(const at::Tensor& t, at::ScalarType type) {
  return at::TensorOptions().dtype(type).device(t.device());
}

// (old_len, new_len, block_table, free_pages, page_size, n_tok, first_pos, stream)
PyObject* kv_layout(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 8, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const at::Tensor& old_len = tensor(a[0], "old_len");
    const int64_t n = old_len.dim() == 1 ? old_len.size(0) : -1;
    fsched_layout_params p{};
    const int32_t* old_p = ints(a[0], n, "old_len");
    const int32_t* new_p = ints(a[1], n, "new_len");
    int32_t* table_p = table(a[2], n, &p.table_width);
    const int32_t* free_p = ints(a[3], -1, "free_pages");
    p.n_free = extent(tensor(a[3], "free_pages").size(0), "free_pages");
    p.n_req = extent(n, "old_len");
    p.page_size = int32(a[4], "page_size");
    p.n_tok = int32(a[5], "n_tok");
    p.first_pos = int32(a[6], "first_pos");
    p.flags = FSCHED_F_DEVICE_PTRS;
    void* stream = handle(a[7]);
    // one allocation holds all results, each from a multiple of 16 bytes on
    const int64_t m = p.n_tok < 0 ? 0 : p.n_tok;
    const int64_t len[5] = {m, m, n + 1, n, 2};
    int64_t at[5], total = 0;
    for (int i = 0; i < 5; ++i) {
      at[i] = total;
      total += (len[i] + 3) & ~(int64_t)3;
    }
    const at::Tensor room = at::empty({total}, like(old_len, at::kInt));
    int32_t* o = (int32_t*)room.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = fsched_kv_layout(&p, old_p, new_p, free_p, table_p, o + at[0], o + at[1], o + at[2],
                          o + at[3], o + at[4], stream);
    Py_END_ALLOW_THREADS;
    check(rc, "fsched_kv_layout");
    PyObject* result = PyTuple_New(5);
    if (!result) throw Raised{};
    for (int i = 0; i < 5; ++i)
      PyTuple_SET_ITEM(result, i, THPVariable_Wrap(room.narrow(0, at[i], len[i])));
    return result;
  });
}

// (qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight, k_weight, eps,
//  interleaved, out, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 12, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache c = cache(a[4], a[5]);
    if (a[2] != Py_None) {  // slots
      written(tensor(a[4], "k_cache"), "k_cache");
      written(tensor(a[5], "v_cache"), "v_cache");
    }
    const int64_t dim = c.c.head_dim;
    const at::Tensor& qkv = rows(a[0], 3, c.type, "qkv");
    const int64_t n = qkv.size(0), heads = qkv.size(1) - 2 * (int64_t)c.c.kv_heads;
    if (heads < 1 || qkv.size(2) != dim || qkv.stride(1) != dim)
      throw Refused{"qkv must be [n_tok, q_heads + 2 kv_heads, head_dim] with heads "
                    "head_dim apart"};
    fsched_rope_params p{};
    const float* cos_sin = nullptr;
    if (a[3] != Py_None) {
      const at::Tensor& t = tensor(a[3], "cos_sin");
      if (t.scalar_type() != at::kFloat || !t.is_cuda() || t.dim() != 2 || !t.is_contiguous())
        throw Refused{"cos_sin must be a contiguous float32 GPU tensor [n_pos, rot_dim]"};
      if (a[1] == Py_None) throw Refused{"a rotation needs positions"};
      cos_sin = (const float*)t.data_ptr();
      p.n_pos = extent(t.size(0), "cos_sin");
      p.rot_dim = extent(t.size(1), "cos_sin");
    }
    const void* weight[2] = {nullptr, nullptr};
    for (int i = 0; i < 2; ++i) {
      if (a[6 + i] == Py_None) continue;
      const char* name = i ? "k_weight" : "q_weight";
      const at::Tensor& w = rows(a[6 + i], 1, c.type, name);
      if (w.size(0) != dim) throw Refused{std::string(name) + " must have head_dim elements"};
      weight[i] = w.data_ptr();
    }
    const at::Tensor out = a[10] == Py_None ? at::empty({n, heads, dim}, like(qkv, c.type))
                                            : rows(a[10], 3, c.type, "out");
    if (out.size(0) != n || out.size(1) != heads || out.size(2) != dim)
      throw Refused{"out must have shape [n_tok, q_heads, head_dim]"};
    written(out, "out");
    p.n_tok = extent(n, "qkv");
    p.q_heads = extent(heads, "qkv");
    p.interleaved = truth(a[9]);
    p.eps = real(a[8]);
    p.flags = FSCHED_F_DEVICE_PTRS;
    p.qkv_stride = qkv.stride(0);
    p.q_token_stride = out.stride(0);
    p.q_head_stride = out.stride(1);
    const int32_t* positions = a[1] == Py_None ? nullptr : ints(a[1], n, "positions");
    const int32_t* slots = a[2] == Py_None ? nullptr : ints(a[2], n, "slots");
    void* stream = handle(a[11]);
    const void* src = qkv.data_ptr();
    void* dst = out.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = fsched_qk_norm_rope(&p, &c.c, src, positions, slots, cos_sin, weight[0], weight[1], dst,
                             stream);
    Py_END_ALLOW_THREADS;
    check(rc, "fsched_qk_norm_rope");
    return THPVariable_Wrap(out);
  });
}

// (q, k_cache, v_cache, prefix_pages, prefix_len, block_table, q_start, kv_len, scale,
//  window, n_sink, max_q, out, return_lse, workspace, stream)
// prefix_pages None: fsched_attend.  workspace None: taken from torch's allocator.
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 16, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const bool shared = a[3] != Py_None;
    const char* name = shared ? "fsched_attend_shared" : "fsched_attend";
    const Cache c = cache(a[1], a[2]);
    const at::Tensor& q = rows(a[0], 3, c.type, "q");
    if (q.size(2) != c.c.head_dim) throw Refused{"q and the cache differ in head_dim"};
    const at::Tensor& kv_len = tensor(a[7], "kv_len");
    const int64_t n = kv_len.dim() == 1 ? kv_len.size(0) : -1;
    fsched_attn_params p{};
    const int32_t* kv_p = ints(a[7], n, "kv_len");
    const int32_t* start_p = ints(a[6], n + 1, "q_start");
    const int32_t* table_p = table(a[5], n, &p.table_width);
    p.prefix_len = int32(a[4], "prefix_len");
    const int32_t* prefix_p = nullptr;
    if (shared) {
      prefix_p = ints(a[3], -1, "prefix_pages");
      if (tensor(a[3], "prefix_pages").size(0) * (int64_t)c.c.page_size < p.prefix_len)
        throw Refused{"prefix_pages must list every page of the prefix"};
    }
    p.n_req = extent(n, "kv_len");
    p.n_tok = extent(q.size(0), "q");
    p.q_heads = extent(q.size(1), "q");
    p.scale = a[8] == Py_None ? 1.0f / std::sqrt((float)c.c.head_dim) : real(a[8]);
    p.window = int32(a[9], "window");
    p.n_sink = int32(a[10], "n_sink");
    p.max_q = a[11] == Py_None ? (p.n_tok > 0 ? p.n_tok : 1) : int32(a[11], "max_q");
    p.flags = FSCHED_F_DEVICE_PTRS;
    const at::Tensor out =
        a[12] == Py_None ? at::empty(q.sizes(), like(q, c.type)) : rows(a[12], 3, c.type, "out");
    if (out.sizes() != q.sizes()) throw Refused{"out and q differ in shape"};
    written(out, "out");
    p.q_token_stride = q.stride(0);
    p.q_head_stride = q.stride(1);
    p.out_token_stride = out.stride(0);
    p.out_head_stride = out.stride(1);
    at::Tensor lse, workspace;
    if (truth(a[13])) lse = at::empty({q.size(0), q.size(1)}, like(q, at::kFloat));
    if (a[14] != Py_None) {
      workspace = tensor(a[14], "workspace");
      if (!workspace.is_cuda() || !workspace.is_contiguous())
        throw Refused{"workspace must be a contiguous GPU tensor"};
    }
    if (!workspace.defined() || workspace.nbytes() == 0) {
      int64_t need = 0;
      check(fsched_attend_workspace(&p, &c.c, &need), name);
      // an empty tensor's address is that of no workspace, which the library would take
      // from its pool
      if (workspace.defined() && need > 0) check(FSCHED_ESCRATCH, name);
      if (need > 0) workspace = at::empty({need}, like(q, at::kByte));
    }
    void* stream = handle(a[15]);
    const void* q_p = q.data_ptr();
    void* out_p = out.data_ptr();
    float* lse_p = lse.defined() ? (float*)lse.data_ptr() : nullptr;
    void* ws = workspace.defined() ? workspace.data_ptr() : nullptr;
    const int64_t ws_bytes = workspace.defined() ? (int64_t)workspace.nbytes() : 0;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = shared ? fsched_attend_shared(&p, &c.c, q_p, prefix_p, table_p, start_p, kv_p, out_p,
                                       lse_p, ws, ws_bytes, stream)
                : fsched_attend(&p, &c.c, q_p, table_p, start_p, kv_p, out_p, lse_p, ws, ws_bytes,
                                stream);
    Py_END_ALLOW_THREADS;
    check(rc, name);
    PyObject* o = THPVariable_Wrap(out);
    if (!lse.defined()) return o;
    PyObject* l = THPVariable_Wrap(lse);
    PyObject* both = PyTuple_Pack(2, o, l);
    Py_XDECREF(o);
    Py_XDECREF(l);
    return both;
  });
}

PyMethodDef methods[] = {
    {"kv_layout", (PyCFunction)(void (*)(void))kv_layout, METH_FASTCALL, nullptr},
    {"qk_norm_rope", (PyCFunction)(void (*)(void))qk_norm_rope, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods,
                      nullptr,               nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
