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

struct Cache4 {
  fsched_kv4_cache c;
  at::ScalarType type;
};

// A cache of 4 bits and the type of the elements beside it.
Cache4 cache4(PyObject* o, at::ScalarType type) {
  const at::Tensor& t = tensor(o, "cache");
  if (t.scalar_type() != at::kByte || !t.is_cuda() || t.dim() != 4 || t.size(3) % 17 != 0 ||
      (t.stride(3) != 1 && t.size(3) > 1))
    throw Refused{"cache must be a uint8 GPU tensor [n_pages, kv_heads, page_size / 16, "
                  "17 head_dim] whose last dimension is contiguous"};
  if (type != at::kBFloat16 && type != at::kHalf)
    throw Refused{"elements beside a cache of 4 bits are bfloat16 or float16"};
  Cache4 r;
  r.type = type;
  r.c = fsched_kv4_cache{};
  r.c.data = t.data_ptr();
  for (int i = 0; i < 3; ++i) r.c.stride[i] = t.stride(i);
  r.c.n_pages = extent(t.size(0), "cache");
  r.c.kv_heads = extent(t.size(1), "cache");
  r.c.page_size = extent(t.size(2) * 16, "cache");
  r.c.head_dim = extent(t.size(3) / 17, "cache");
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

// Two tensors as a tuple.
PyObject* pair(const at::Tensor& x, const at::Tensor& y) {
  PyObject* a = THPVariable_Wrap(x);
  PyObject* b = THPVariable_Wrap(y);
  PyObject* both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  if (!both) throw Raised{};
  return both;
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

// The rotation's arguments but for the cache, from a[0] on; those behind the cache (q_weight,
// k_weight, eps, interleaved, out, stream) from a[rest] on.
template <class C, class Call>
PyObject* rope(PyObject* const* a, int rest, const C& c, const char* name, Call call) {
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
    if (a[rest + i] == Py_None) continue;
    const char* which = i ? "k_weight" : "q_weight";
    const at::Tensor& w = rows(a[rest + i], 1, c.type, which);
    if (w.size(0) != dim) throw Refused{std::string(which) + " must have head_dim elements"};
    weight[i] = w.data_ptr();
  }
  const at::Tensor out = a[rest + 4] == Py_None ? at::empty({n, heads, dim}, like(qkv, c.type))
                                                : rows(a[rest + 4], 3, c.type, "out");
  if (out.size(0) != n || out.size(1) != heads || out.size(2) != dim)
    throw Refused{"out must have shape [n_tok, q_heads, head_dim]"};
  written(out, "out");
  p.n_tok = extent(n, "qkv");
  p.q_heads = extent(heads, "qkv");
  p.interleaved = truth(a[rest + 3]);
  p.eps = real(a[rest + 2]);
  p.flags = FSCHED_F_DEVICE_PTRS;
  p.qkv_stride = qkv.stride(0);
  p.q_token_stride = out.stride(0);
  p.q_head_stride = out.stride(1);
  const int32_t* positions = a[1] == Py_None ? nullptr : ints(a[1], n, "positions");
  const int32_t* slots = a[2] == Py_None ? nullptr : ints(a[2], n, "slots");
  void* stream = handle(a[rest + 5]);
  const void* src = qkv.data_ptr();
  void* dst = out.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call(&p, &c.c, src, positions, slots, cos_sin, weight[0], weight[1], dst, stream);
  Py_END_ALLOW_THREADS;
  check(rc, name);
  return THPVariable_Wrap(out);
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
    return rope(a, 6, c, "fsched_qk_norm_rope", fsched_qk_norm_rope);
  });
}

// The type of the elements beside a cache of 4 bits: that of a call's rows.
at::ScalarType type_of(PyObject* o, const char* name) {
  return tensor(o, name).scalar_type();
}

// (qkv, positions, slots, cos_sin, cache, q_weight, k_weight, eps, interleaved, out, stream)
PyObject* qk_norm_rope4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 11, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache4 c = cache4(a[4], type_of(a[0], "qkv"));
    if (a[2] != Py_None) written(tensor(a[4], "cache"), "cache");
    return rope(a, 5, c, "fsched_qk_norm_rope4", fsched_qk_norm_rope4);
  });
}

// (cache, slots, f16, stream)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 4, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache4 c = cache4(a[0], truth(a[2]) ? at::kHalf : at::kBFloat16);
    const int32_t* slots = ints(a[1], -1, "slots");
    const int64_t n = tensor(a[1], "slots").size(0);
    fsched_read_params p{};
    p.n_tok = extent(n, "slots");
    p.flags = FSCHED_F_DEVICE_PTRS;
    p.token_stride = (int64_t)c.c.kv_heads * c.c.head_dim;
    p.head_stride = c.c.head_dim;
    void* stream = handle(a[3]);
    const at::Tensor both =
        at::empty({2, n, c.c.kv_heads, c.c.head_dim}, like(tensor(a[0], "cache"), c.type));
    char* k = (char*)both.data_ptr();
    char* v = k + both.nbytes() / 2;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = fsched_kv4_read(&p, &c.c, slots, k, v, stream);
    Py_END_ALLOW_THREADS;
    check(rc, "fsched_kv4_read");
    return pair(both.select(0, 0), both.select(0, 1));
  });
}

// What the attention calls have in common: their parameters and index arrays.
struct Step {
  fsched_attn_params p;
  const int32_t *table, *q_start, *kv_len, *prefix;
};

// q, then from a[at] on: block_table, q_start, kv_len; from a[opt] on: scale, window, n_sink,
// max_q; and the prefix (pages or None, length).
template <class C>
Step step_of(PyObject* const* a, int at, int opt, PyObject* pages, PyObject* prefix_len,
             const C& c, const at::Tensor& q) {
  if (q.size(2) != c.c.head_dim) throw Refused{"q and the cache differ in head_dim"};
  Step s{};
  fsched_attn_params& p = s.p;
  const at::Tensor& kv_len = tensor(a[at + 2], "kv_len");
  const int64_t n = kv_len.dim() == 1 ? kv_len.size(0) : -1;
  s.kv_len = ints(a[at + 2], n, "kv_len");
  s.q_start = ints(a[at + 1], n + 1, "q_start");
  s.table = table(a[at], n, &p.table_width);
  p.prefix_len = int32(prefix_len, "prefix_len");
  if (pages != Py_None) {
    s.prefix = ints(pages, -1, "prefix_pages");
    if (tensor(pages, "prefix_pages").size(0) * (int64_t)c.c.page_size < p.prefix_len)
      throw Refused{"prefix_pages must list every page of the prefix"};
  }
  p.n_req = extent(n, "kv_len");
  p.n_tok = extent(q.size(0), "q");
  p.q_heads = extent(q.size(1), "q");
  p.scale = a[opt] == Py_None ? 1.0f / std::sqrt((float)c.c.head_dim) : real(a[opt]);
  p.window = int32(a[opt + 1], "window");
  p.n_sink = int32(a[opt + 2], "n_sink");
  p.max_q = a[opt + 3] == Py_None ? (p.n_tok > 0 ? p.n_tok : 1) : int32(a[opt + 3], "max_q");
  p.flags = FSCHED_F_DEVICE_PTRS;
  p.q_token_stride = q.stride(0);
  p.q_head_stride = q.stride(1);
  return s;
}

// Attention with its outputs; a[out] on: out, return_lse, workspace, stream.
template <class C, class Size, class Call>
PyObject* attention(PyObject* const* a, int out_at, const at::Tensor& q, Step& s, const C& c,
                    const char* name, Size size, Call call) {
  fsched_attn_params& p = s.p;
  const at::Tensor out = a[out_at] == Py_None ? at::empty(q.sizes(), like(q, c.type))
                                              : rows(a[out_at], 3, c.type, "out");
  if (out.sizes() != q.sizes()) throw Refused{"out and q differ in shape"};
  written(out, "out");
  p.out_token_stride = out.stride(0);
  p.out_head_stride = out.stride(1);
  at::Tensor lse, workspace;
  if (truth(a[out_at + 1])) lse = at::empty({q.size(0), q.size(1)}, like(q, at::kFloat));
  if (a[out_at + 2] != Py_None) {
    workspace = tensor(a[out_at + 2], "workspace");
    if (!workspace.is_cuda() || !workspace.is_contiguous())
      throw Refused{"workspace must be a contiguous GPU tensor"};
  }
  if (!workspace.defined() || workspace.nbytes() == 0) {
    int64_t need = 0;
    check(size(&p, &c.c, &need), name);
    // an empty tensor's address is that of no workspace, which the library would take
    // from its pool
    if (workspace.defined() && need > 0) check(FSCHED_ESCRATCH, name);
    if (need > 0) workspace = at::empty({need}, like(q, at::kByte));
  }
  void* stream = handle(a[out_at + 3]);
  const void* q_p = q.data_ptr();
  void* out_p = out.data_ptr();
  float* lse_p = lse.defined() ? (float*)lse.data_ptr() : nullptr;
  void* ws = workspace.defined() ? workspace.data_ptr() : nullptr;
  const int64_t ws_bytes = workspace.defined() ? (int64_t)workspace.nbytes() : 0;
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call(&p, &c.c, q_p, out_p, lse_p, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS;
  check(rc, name);
  return lse.defined() ? pair(out, lse) : THPVariable_Wrap(out);
}

// (q, k_cache, v_cache, prefix_pages, prefix_len, block_table, q_start, kv_len, scale,
//  window, n_sink, max_q, out, return_lse, workspace, stream)
// prefix_pages None: fsched_attend.  workspace None: taken from torch's allocator.
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 16, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const bool shared = a[3] != Py_None;
    const Cache c = cache(a[1], a[2]);
    const at::Tensor& q = rows(a[0], 3, c.type, "q");
    Step s = step_of(a, 5, 8, a[3], a[4], c, q);
    return attention(
        a, 12, q, s, c, shared ? "fsched_attend_shared" : "fsched_attend",
        fsched_attend_workspace,
        [&](const fsched_attn_params* p, const fsched_kv_cache* kv, const void* q_p, void* out,
            float* lse, void* ws, int64_t bytes, void* stream) {
          return shared ? fsched_attend_shared(p, kv, q_p, s.prefix, s.table, s.q_start, s.kv_len,
                                               out, lse, ws, bytes, stream)
                        : fsched_attend(p, kv, q_p, s.table, s.q_start, s.kv_len, out, lse, ws,
                                        bytes, stream);
        });
  });
}

// (q, cache, prefix_pages, prefix_len, block_table, q_start, kv_len, scale, window, n_sink,
//  max_q, out, return_lse, workspace, stream)
PyObject* attend4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 15, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache4 c = cache4(a[1], type_of(a[0], "q"));
    const at::Tensor& q = rows(a[0], 3, c.type, "q");
    Step s = step_of(a, 4, 7, a[2], a[3], c, q);
    if (!s.prefix && s.p.prefix_len != 0) throw Refused{"a prefix needs prefix_pages"};
    return attention(
        a, 11, q, s, c, "fsched_attend4", fsched_attend4_workspace,
        [&](const fsched_attn_params* p, const fsched_kv4_cache* kv, const void* q_p, void* out,
            float* lse, void* ws, int64_t bytes, void* stream) {
          return fsched_attend4(p, kv, q_p, s.prefix, s.table, s.q_start, s.kv_len, out, lse, ws,
                                bytes, stream);
        });
  });
}

// Weights of held tokens; a[1] is lse, a[at] on: block_table, q_start, kv_len, weight, scale,
// window, n_sink, max_q, prefix_len, stream.
template <class C, class Size, class Call>
PyObject* weights(PyObject* const* a, int at, const C& c, const char* name, Size size, Call call) {
  const at::Tensor& q = rows(a[0], 3, c.type, "q");
  Step s = step_of(a, at, at + 4, Py_None, a[at + 8], c, q);
  const at::Tensor& lse = tensor(a[1], "lse");
  if (lse.scalar_type() != at::kFloat || !lse.is_cuda() || lse.dim() != 2 ||
      !lse.is_contiguous() || lse.size(0) != q.size(0) || lse.size(1) != q.size(1))
    throw Refused{"lse must be a contiguous float32 GPU tensor [n_tok, q_heads]"};
  const at::Tensor& weight = tensor(a[at + 3], "weight");
  const int64_t row = (int64_t)s.p.table_width * c.c.page_size;
  if (weight.scalar_type() != at::kFloat || !weight.is_cuda() || weight.dim() != 2 ||
      weight.size(0) != s.p.n_req || weight.size(1) != row ||
      (weight.stride(1) != 1 && row > 1) || (weight.stride(0) < row && s.p.n_req > 1))
    throw Refused{"weight must be a float32 GPU tensor [n_req, table width * page_size] whose "
                  "rows are contiguous and apart"};
  const int64_t stride = weight.size(0) > 1 ? weight.stride(0) : row;
  int64_t need = 0;
  check(size(&s.p, &c.c, &need), name);
  at::Tensor workspace;
  if (need > 0) workspace = at::empty({need}, like(q, at::kByte));
  void* ws = workspace.defined() ? workspace.data_ptr() : nullptr;
  void* stream = handle(a[at + 9]);
  const void* q_p = q.data_ptr();
  const float* lse_p = (const float*)lse.data_ptr();
  float* w_p = (float*)weight.data_ptr();
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call(&s.p, &c.c, q_p, lse_p, s.table, s.q_start, s.kv_len, w_p, stride, ws, need, stream);
  Py_END_ALLOW_THREADS;
  check(rc, name);
  Py_INCREF(a[at + 3]);
  return a[at + 3];
}

// (q, lse, k_cache, block_table, q_start, kv_len, weight, scale, window, n_sink, max_q,
//  prefix_len, stream)
PyObject* attend_weight(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache c = cache(a[2], a[2]);
    return weights(a, 3, c, "fsched_attend_weight", fsched_attend_weight_workspace,
                   fsched_attend_weight);
  });
}

// The same with a cache of 4 bits.
PyObject* attend4_weight(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 13, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const Cache4 c = cache4(a[2], type_of(a[0], "q"));
    return weights(a, 3, c, "fsched_attend4_weight", fsched_attend4_weight_workspace,
                   fsched_attend4_weight);
  });
}

// (weight, kv_len, block_table, budget, page_size, n_sink, n_recent, n_freed, stream)
PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 9, [&]() -> PyObject* {
    const c10::DeviceGuard on = one_device(a, n_args);
    const at::Tensor& kv_len = tensor(a[1], "kv_len");
    const int64_t n = kv_len.dim() == 1 ? kv_len.size(0) : -1;
    fsched_evict_params p{};
    const int32_t* kv_p = ints(a[1], n, "kv_len");
    const int32_t* table_p = table(a[2], n, &p.table_width);
    const int32_t* budget_p = ints(a[3], n, "budget");
    p.n_req = extent(n, "kv_len");
    p.page_size = int32(a[4], "page_size");
    p.n_sink = int32(a[5], "n_sink");
    p.n_recent = int32(a[6], "n_recent");
    const int64_t width = p.table_width, row = width * p.page_size;
    // no more pages than the table has can be given up
    p.n_freed = a[7] == Py_None ? extent(n * width, "block_table") : int32(a[7], "n_freed");
    p.flags = FSCHED_F_DEVICE_PTRS;
    const at::Tensor& weight = tensor(a[0], "weight");
    if (weight.scalar_type() != at::kFloat || !weight.is_cuda() || weight.dim() != 2 ||
        weight.size(0) != n || weight.size(1) != row || (weight.stride(1) != 1 && row > 1))
      throw Refused{"weight must be a float32 GPU tensor [n_req, table width * page_size] whose "
                    "rows are contiguous"};
    p.weight_stride = n > 1 ? weight.stride(0) : row;
    void* stream = handle(a[8]);
    int64_t need = 0;
    check(fsched_kv_evict_workspace(&p, &need), "fsched_kv_evict");
    // one allocation holds the whole numbers, each from a multiple of 16 bytes on
    const int64_t len[4] = {n * width, n, p.n_freed, 1};
    int64_t at[4], total = 0;
    for (int i = 0; i < 4; ++i) {
      at[i] = total;
      total += (len[i] + 3) & ~(int64_t)3;
    }
    const at::Tensor room = at::empty({total}, like(kv_len, at::kInt));
    const at::Tensor moved = at::empty({n, row}, like(kv_len, at::kFloat));
    at::Tensor workspace;
    if (need > 0) workspace = at::empty({need}, like(kv_len, at::kByte));
    void* ws = workspace.defined() ? workspace.data_ptr() : nullptr;
    int32_t* o = (int32_t*)room.data_ptr();
    const float* w_p = (const float*)weight.data_ptr();
    float* moved_p = (float*)moved.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = fsched_kv_evict(&p, w_p, kv_p, table_p, budget_p, o + at[0], moved_p, o + at[1],
                         o + at[2], o + at[3], ws, need, stream);
    Py_END_ALLOW_THREADS;
    check(rc, "fsched_kv_evict");
    const at::Tensor out[5] = {room.narrow(0, at[0], len[0]).view({n, width}), moved,
                               room.narrow(0, at[1], n), room.narrow(0, at[2], len[2]),
                               room.narrow(0, at[3], 1)};
    PyObject* result = PyTuple_New(5);
    if (!result) throw Raised{};
    for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(result, i, THPVariable_Wrap(out[i]));
    return result;
  });
}

PyMethodDef methods[] = {
    {"kv_layout", (PyCFunction)(void (*)(void))kv_layout, METH_FASTCALL, nullptr},
    {"qk_norm_rope", (PyCFunction)(void (*)(void))qk_norm_rope, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {"qk_norm_rope4", (PyCFunction)(void (*)(void))qk_norm_rope4, METH_FASTCALL, nullptr},
    {"kv4_read", (PyCFunction)(void (*)(void))kv4_read, METH_FASTCALL, nullptr},
    {"attend4", (PyCFunction)(void (*)(void))attend4, METH_FASTCALL, nullptr},
    {"attend_weight", (PyCFunction)(void (*)(void))attend_weight, METH_FASTCALL, nullptr},
    {"attend4_weight", (PyCFunction)(void (*)(void))attend4_weight, METH_FASTCALL, nullptr},
    {"kv_evict", (PyCFunction)(void (*)(void))kv_evict, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods,
                      nullptr,               nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
