// The calls of poss_paged.h over torch tensors, as a Python module: checks of the tensors, outputs and scratch from torch's
// allocator, the call on torch's current stream.  paged.py gives them their signatures.
//
// Why not ctypes like the calls of poss.h: those run for hundreds of microseconds on the GPU, most of these for 2 to 20, and a
// loop of small calls runs at the speed of the host.  Checks in Python with a ctypes call took 8.8 us for a commit, 20 us for a
// remapping or a beam step and 23 us for an append with its attention, mostly attribute reads and argument conversions; here
// they take 3.8, 11 and 10 us, the kernels' launches among them.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <climits>
#include <string>
#include "../../include/poss_paged.h"

namespace {

using at::IntArrayRef;
using at::ScalarType;
using at::Tensor;

struct Refused {};                      // a Python error is set
PyObject* g_error = nullptr;            // the binding's PossError

[[noreturn]] void refuse(const std::string& text) {
  PyErr_SetString(PyExc_ValueError, text.c_str());
  throw Refused();
}
std::string type_name(ScalarType t) {
  switch (t) {
    case at::kInt: return "torch.int32";
    case at::kLong: return "torch.int64";
    case at::kFloat: return "torch.float32";
    case at::kBFloat16: return "torch.bfloat16";
    case at::kByte: return "torch.uint8";
    default: return c10::toString(t);
  }
}
std::string list(IntArrayRef x) {
  std::string s = "[";
  for (size_t i = 0; i < x.size(); ++i) s += (i ? ", " : "") + std::to_string(x[i]);
  return s + "]";
}
const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": a CUDA tensor is wanted, got " + Py_TYPE(o)->tp_name);
  const Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided) refuse(std::string(name) + ": a dense tensor is wanted");
  return t;
}
[[noreturn]] void wrong(const Tensor& t, ScalarType type, IntArrayRef shape, const char* name, int dev) {
  refuse(std::string(name) + ": a contiguous " + type_name(type) + " tensor " + list(shape) + " on cuda:" + std::to_string(dev) +
         " is wanted, got " + type_name(t.scalar_type()) + " " + list(t.sizes()) + " on " + t.device().str() +
         (t.is_contiguous() ? "" : ", not contiguous"));
}
bool on(const Tensor& t, int dev) { return t.is_cuda() && t.get_device() == dev; }
// address of a contiguous tensor of the given type and shape on device `dev`
void* arg(PyObject* o, ScalarType type, IntArrayRef shape, const char* name, int dev) {
  const Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.sizes() != shape || !on(t, dev) || !t.is_contiguous()) wrong(t, type, shape, name, dev);
  return t.data_ptr();
}
void* opt(PyObject* o, ScalarType type, IntArrayRef shape, const char* name, int dev) {
  return o == Py_None ? nullptr : arg(o, type, shape, name, dev);
}
template <class T> T* ints(PyObject* o, IntArrayRef shape, const char* name, int dev) {
  return static_cast<T*>(arg(o, sizeof(T) == 4 ? at::kInt : at::kLong, shape, name, dev));
}
int32_t* opt_ints(PyObject* o, IntArrayRef shape, const char* name, int dev) {
  return static_cast<int32_t*>(opt(o, at::kInt, shape, name, dev));
}
int small(int64_t x) {
  if (x > INT_MAX) refuse("a dimension does not fit 32 bits");
  return (int)x;
}
int integer(PyObject* o) {
  const long x = PyLong_AsLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused();
  if (x < INT_MIN || x > INT_MAX) refuse("an integer argument does not fit 32 bits");
  return (int)x;
}
int current(const Tensor& t, const char* name) {
  if (!t.is_cuda() || t.get_device() != c10::cuda::current_device())
    refuse(std::string(name) + ": a tensor on the current device is wanted, got one on " + t.device().str());
  return t.get_device();
}
bool pool_type(ScalarType t) { return t == at::kBFloat16 || t == at::kFloat; }

struct Pool {
  poss_page_pool p;
  void* pages;
  int dev;
  ScalarType type;
  explicit Pool(PyObject* o) {
    const Tensor& t = tensor(o, "kv_pages");
    if (t.dim() != 6 || !t.is_contiguous()) refuse("kv_pages: a contiguous CUDA tensor of six dimensions is wanted");
    type = t.scalar_type();
    if (t.size(2) != 2 || !pool_type(type))
      refuse("kv_pages: [layers][pages][2][kv heads][page slots][head dim] of bf16 or fp32 is wanted, got " + type_name(type) + " " +
             list(t.sizes()));
    dev = current(t, "kv_pages");
    p = {small(t.size(0)), small(t.size(1)), small(t.size(3)), small(t.size(4)), small(t.size(5)),
         type == at::kBFloat16 ? POSS_BF16 : POSS_FP32};
    pages = t.data_ptr();
  }
};
struct Table {
  int32_t* at;
  int n, max_pages;
  Table(PyObject* o, const char* name, int dev) {
    const Tensor& t = tensor(o, name);
    if (t.dim() != 2) refuse(std::string(name) + ": [sequences][max pages] is wanted");
    n = small(t.size(0));
    max_pages = small(t.size(1));
    at = ints<int32_t>(o, t.sizes(), name, dev);
  }
};
// [batch][rows][heads][d] whose rows may lie apart (a slice of a fused projection)
struct Rows {
  void* at;
  int64_t ld;
  int batch, rows, heads;
  Rows(PyObject* o, const char* name, int64_t want_heads, const Pool& pool) {
    const Tensor& t = tensor(o, name);
    if (t.dim() != 4) refuse(std::string(name) + ": [batch][rows][heads][head dim] is wanted");
    const int64_t b = t.size(0), r = t.size(1), h = t.size(2), d = pool.p.head_dim;
    if (t.scalar_type() != pool.type || t.size(3) != d || (want_heads >= 0 && h != want_heads) || !on(t, pool.dev))
      wrong(t, pool.type, {b, r, want_heads >= 0 ? want_heads : h, d}, name, pool.dev);
    batch = small(b);
    rows = small(r);
    heads = small(h);
    at = t.data_ptr();
    ld = h * d;
    if (t.is_contiguous()) return;
    if (r > 1) ld = t.stride(1);
    else if (b > 1) ld = t.stride(0);
    if (t.stride(3) != 1 || (h > 1 && t.stride(2) != d) || (r > 1 && b > 1 && t.stride(0) != r * ld) || ld < h * d)
      refuse(std::string(name) + ": heads contiguous and rows evenly apart are wanted, got strides " + list(t.strides()));
  }
};
Tensor fresh(IntArrayRef shape, ScalarType type, int dev) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, dev));
}
// the caller's scratch, or some for the call (its memory is this stream's again behind it)
struct Scratch {
  Tensor own;
  void* at;
  size_t bytes;
  Scratch(PyObject* o, size_t need, int dev) {
    if (o == Py_None) {
      own = fresh({(int64_t)need}, at::kByte, dev);
      at = own.data_ptr();
      bytes = need;
      return;
    }
    const Tensor& t = tensor(o, "workspace");
    if (!on(t, dev) || t.scalar_type() != at::kByte || !t.is_contiguous())
      refuse("workspace: a contiguous uint8 tensor on cuda:" + std::to_string(dev) + " is wanted");
    at = t.data_ptr();
    bytes = (size_t)t.numel();
  }
};
// f(stream) on the device's current stream, without the interpreter's lock: f must not throw
template <class F> void call(const char* where, int dev, F f) {
  const poss_stream stream = reinterpret_cast<poss_stream>(c10::cuda::getCurrentCUDAStream(dev).stream());
  int code;
  Py_BEGIN_ALLOW_THREADS
  code = f(stream);
  Py_END_ALLOW_THREADS
  if (code) {
    PyObject* e = PyObject_CallFunction(g_error, "is", code, where);
    if (e) {
      PyErr_SetObject(g_error, e);
      Py_DECREF(e);
    }
    throw Refused();
  }
}
// a dict of outputs: the caller's, or one that is filled here
struct Outputs {
  PyObject* dict;                       // a new reference
  bool made;
  explicit Outputs(PyObject* o) : dict(o), made(o == Py_None) {
    if (made) {
      dict = PyDict_New();
      if (!dict) throw Refused();
    } else {
      if (!PyDict_Check(o)) refuse("out: a dict of tensors is wanted");
      Py_INCREF(dict);
    }
  }
  ~Outputs() { Py_XDECREF(dict); }
  PyObject* release() {
    PyObject* d = dict;
    dict = nullptr;
    return d;
  }
  void* get(const char* key, ScalarType type, IntArrayRef shape, const char* name, int dev) {
    if (made) {
      Tensor t = fresh(shape, type, dev);
      void* p = t.data_ptr();
      PyObject* o = THPVariable_Wrap(std::move(t));
      const int bad = !o || PyDict_SetItemString(dict, key, o);
      Py_XDECREF(o);
      if (bad) throw Refused();
      return p;
    }
    PyObject* o = PyDict_GetItemString(dict, key);
    if (!o) refuse(std::string("out: no tensor for ") + key);
    return arg(o, type, shape, name, dev);
  }
};

// Every function takes its arguments by place, as paged.py passes them.
#define POSS_CALL(name, count)                                                                          \
  PyObject* name##_body(PyObject* const* x);                                                            \
  PyObject* name(PyObject*, PyObject* const* x, Py_ssize_t n) {                                         \
    HANDLE_TH_ERRORS                                                                                    \
    if (n != count) {                                                                                   \
      PyErr_SetString(PyExc_TypeError, #name ": " #count " arguments");                                 \
      return nullptr;                                                                                   \
    }                                                                                                   \
    try {                                                                                               \
      return name##_body(x);                                                                            \
    } catch (const Refused&) {                                                                          \
      return nullptr;                                                                                   \
    }                                                                                                   \
    END_HANDLE_TH_ERRORS                                                                                \
  }                                                                                                     \
  PyObject* name##_body(PyObject* const* x)

POSS_CALL(append, 8) {  // k, v, kv_pages, layer, tables, prefix_len, n_rows, status
  const Pool pool(x[2]);
  const int dev = pool.dev;
  const Rows k(x[0], "k", pool.p.n_kv_heads, pool), v(x[1], "v", pool.p.n_kv_heads, pool);
  if (v.ld != k.ld || v.batch != k.batch || v.rows != k.rows) refuse("k and v: the same shape and the same strides are wanted");
  const Table t(x[4], "tables", dev);
  if (t.n != k.batch) wrong(tensor(x[4], "tables"), at::kInt, {k.batch, t.max_pages}, "tables", dev);
  const int layer = integer(x[3]);
  const int32_t* prefix = ints<int32_t>(x[5], {k.batch}, "prefix_len", dev);
  const int32_t* n_rows = opt_ints(x[6], {k.batch}, "n_rows", dev);
  int32_t* status = opt_ints(x[7], {1}, "status", dev);
  call("poss_pages_append", dev, [&](poss_stream stream) {
    return poss_pages_append(&pool.p, layer, pool.pages, t.at, t.max_pages, k.batch, k.rows, k.at, v.at, k.ld, prefix, n_rows, status,
                             stream);
  });
  Py_RETURN_NONE;
}

POSS_CALL(attention, 11) {  // q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows, out, workspace, status
  const Pool pool(x[1]);
  const int dev = pool.dev;
  const Rows q(x[0], "q", -1, pool);
  const int b = q.batch, r = q.rows;
  const int64_t shape[4] = {b, r, q.heads, pool.p.head_dim};
  const double scale = PyFloat_AsDouble(x[6]);
  if (scale == -1.0 && PyErr_Occurred()) throw Refused();
  Tensor made;
  void* out;
  if (x[8] == Py_None) {
    made = fresh(shape, pool.type, dev);
    out = made.data_ptr();
  } else {
    out = arg(x[8], pool.type, shape, "out", dev);
  }
  if (b && r) {
    const Table t(x[3], "tables", dev);
    if (t.n != b) wrong(tensor(x[3], "tables"), at::kInt, {b, t.max_pages}, "tables", dev);
    const int layer = integer(x[2]);
    const int32_t* prefix = ints<int32_t>(x[4], {b}, "prefix_len", dev);
    const int32_t* n_rows = opt_ints(x[7], {b}, "n_rows", dev);
    const int64_t* mask = ints<int64_t>(x[5], {b, r, (r + 63) / 64}, "anc_mask", dev);
    int32_t* status = opt_ints(x[10], {1}, "status", dev);
    const Scratch ws(x[9], poss_paged_attention_workspace_bytes(&pool.p, b, r, q.heads, t.max_pages), dev);
    call("poss_paged_tree_attention", dev, [&](poss_stream stream) {
      return poss_paged_tree_attention(&pool.p, layer, pool.pages, t.at, t.max_pages, b, r, q.heads, q.at, q.ld, prefix, n_rows,
                                       reinterpret_cast<const uint64_t*>(mask), (float)scale, out, ws.at, ws.bytes, status,
                                       stream);
    });
  }
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[8]);
  return x[8];
}

POSS_CALL(compact, 7) {  // kv_pages, tables, prefix_len, path, n_accepted, out_len, status
  const Pool pool(x[0]);
  const int dev = pool.dev;
  const Table t(x[1], "tables", dev);
  const int b = t.n;
  const int32_t* prefix = ints<int32_t>(x[2], {b}, "prefix_len", dev);
  const int32_t* path = ints<int32_t>(x[3], {b, POSS_MAX_DEPTH + 1}, "path", dev);
  const int32_t* accepted = ints<int32_t>(x[4], {b}, "n_accepted", dev);
  int32_t* status = opt_ints(x[6], {1}, "status", dev);
  Tensor made;
  int32_t* out;
  if (x[5] == Py_None) {
    made = fresh({b}, at::kInt, dev);
    out = static_cast<int32_t*>(made.data_ptr());
  } else {
    out = ints<int32_t>(x[5], {b}, "out_len", dev);
  }
  call("poss_pages_compact", dev, [&](poss_stream stream) {
    return poss_pages_compact(&pool.p, pool.pages, t.at, t.max_pages, b, prefix, path, accepted, out, status, stream);
  });
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[5]);
  return x[5];
}

POSS_CALL(remap, 9) {  // kv_pages, tables, seq_len, refs, parents, room, out, workspace, status
  const Pool pool(x[0]);
  const int dev = pool.dev;
  const Table t(x[1], "tables", dev);
  const int n0 = t.n, pages = pool.p.n_pages;
  int n1 = n0;
  if (x[4] != Py_None) n1 = small(tensor(x[4], "parents").numel());
  const int32_t* parents = opt_ints(x[4], {n1}, "parents", dev);
  const int32_t* room = opt_ints(x[5], {n1}, "room", dev);
  const int32_t* len = ints<int32_t>(x[2], {n0}, "seq_len", dev);
  const int32_t* refs = ints<int32_t>(x[3], {pages}, "refs", dev);
  int32_t* status = opt_ints(x[8], {1}, "status", dev);
  Outputs out(x[6]);
  auto get = [&](const char* key, IntArrayRef shape, const char* name) {
    return static_cast<int32_t*>(out.get(key, at::kInt, shape, name, dev));
  };
  int32_t* out_tables = get("tables", {n1, t.max_pages}, "out tables");
  int32_t* out_refs = get("refs", {pages}, "out refs");
  int32_t* out_len = get("seq_len", {n1}, "out seq_len");
  int32_t* n_free = get("n_free", {1}, "n_free");
  const Scratch ws(x[7], poss_pages_remap_workspace_bytes(&pool.p, n0, n1, t.max_pages), dev);
  // (tables made here hold whatever their memory held: never pages that somebody might write to)
  const auto remap = out.made ? poss_pages_remap_fresh : poss_pages_remap;
  call("poss_pages_remap", dev, [&](poss_stream stream) {
    return remap(&pool.p, pool.pages, t.at, out_tables, t.max_pages, n0, n1, len, refs, out_refs, parents, room, out_len, n_free, ws.at,
                 ws.bytes, status, stream);
  });
  return out.release();
}

POSS_CALL(beam_select, 6) {  // logits, scores, finished, eos, out, workspace
  const Tensor& logits = tensor(x[0], "logits");
  if (logits.dim() != 3 || !pool_type(logits.scalar_type()))
    refuse("logits: a CUDA tensor [batch][beams][vocab] of fp32 or bf16 is wanted");
  const int dev = current(logits, "logits");
  const int b = small(logits.size(0)), k = small(logits.size(1)), vocab = small(logits.size(2));
  if (!logits.is_contiguous()) wrong(logits, logits.scalar_type(), logits.sizes(), "logits", dev);
  const int64_t shape[2] = {b, k};
  const float* scores = static_cast<float*>(arg(x[1], at::kFloat, shape, "scores", dev));
  const int32_t* finished = opt_ints(x[2], shape, "finished", dev);
  const int eos = integer(x[3]);
  Outputs out(x[4]);
  auto get = [&](const char* key, ScalarType type, const char* name) { return out.get(key, type, shape, name, dev); };
  int32_t* tokens = static_cast<int32_t*>(get("tokens", at::kInt, "out tokens"));
  int32_t* parents = static_cast<int32_t*>(get("parents", at::kInt, "out parents"));
  float* out_scores = static_cast<float*>(get("scores", at::kFloat, "out scores"));
  int32_t* done = static_cast<int32_t*>(get("finished", at::kInt, "out finished"));
  const Scratch ws(x[5], poss_beam_select_workspace_bytes(b, k, vocab), dev);
  call("poss_beam_select", dev, [&](poss_stream stream) {
    return poss_beam_select(logits.data_ptr(), logits.scalar_type() == at::kBFloat16 ? POSS_BF16 : POSS_FP32, b, k, vocab, scores,
                            finished, eos, tokens, parents, out_scores, done, ws.at, ws.bytes, stream);
  });
  return out.release();
}

PyObject* bind(PyObject*, PyObject* error) {  // the exception that a refused call raises: error(code, name of the call)
  Py_INCREF(error);
  Py_XSETREF(g_error, error);
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"append", FAST(append)},           {"attention", FAST(attention)}, {"compact", FAST(compact)},
                         {"remap", FAST(remap)},             {"beam_select", FAST(beam_select)},
                         {"bind", bind, METH_O, nullptr},    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_calls() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_with_torch", POSS_BUILT_WITH_TORCH)) Py_CLEAR(m);
  return m;
}
