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
    case at::kDouble: return "torch.float64";
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
  Rows(PyObject* o, const char* name, int64_t want_heads, const Pool& pool) : Rows(o, name, want_heads, pool.p.head_dim, pool.type, pool.dev) {}
  Rows(PyObject* o, const char* name, int64_t want_heads, int64_t d, ScalarType type, int dev) {
    const Tensor& t = tensor(o, name);
    if (t.dim() != 4) refuse(std::string(name) + ": [batch][rows][heads][head dim] is wanted");
    const int64_t b = t.size(0), r = t.size(1), h = t.size(2);
    if (t.scalar_type() != type || t.size(3) != d || (want_heads >= 0 && h != want_heads) || !on(t, dev))
      wrong(t, type, {b, r, want_heads >= 0 ? want_heads : h, d}, name, dev);
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
// the slots' attention weights [layers][batch][kv heads][slots]
struct Mass {
  float* at;
  int64_t slots;
  Mass(PyObject* o, const char* name, const Pool& pool, int batch) {
    const Tensor& t = tensor(o, name);
    if (t.dim() != 4) refuse(std::string(name) + ": [layers][batch][kv heads][slots] is wanted");
    slots = t.size(3);
    at = static_cast<float*>(arg(o, at::kFloat, {pool.p.n_layers, batch, pool.p.n_kv_heads, slots}, name, pool.dev));
  }
};
double real(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Refused();
  return x;
}
int truth(PyObject* o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw Refused();
  return x;
}
// radians per position, of rot_dim / 2 pairs
struct Frequencies {
  const double* at;
  int rot_dim;
  Frequencies(PyObject* o, int dev) {
    const Tensor& t = tensor(o, "freq");
    if (t.dim() != 1) refuse("freq: a tensor of one dimension is wanted");
    at = static_cast<const double*>(arg(o, at::kDouble, t.sizes(), "freq", dev));
    if (t.numel() > INT_MAX / 2) refuse("freq: too many pairs");
    rot_dim = 2 * (int)t.numel();
  }
};
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
  const double scale = real(x[6]);
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

POSS_CALL(compact, 8) {  // kv_pages, tables, prefix_len, path, n_accepted, out_len, status, mass
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
  if (x[7] == Py_None) {
    call("poss_pages_compact", dev, [&](poss_stream stream) {
      return poss_pages_compact(&pool.p, pool.pages, t.at, t.max_pages, b, prefix, path, accepted, out, status, stream);
    });
  } else {
    const Mass mass(x[7], "mass", pool, b);
    call("poss_pages_compact_mass", dev, [&](poss_stream stream) {
      return poss_pages_compact_mass(&pool.p, pool.pages, mass.at, mass.slots, t.at, t.max_pages, b, prefix, path, accepted, out, status,
                                     stream);
    });
  }
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

POSS_CALL(rotary, 6) {  // x, positions, freq, out, interleaved, magnitude
  const Tensor& t = tensor(x[0], "x");
  if (t.dim() != 4 || !pool_type(t.scalar_type())) refuse("x: a CUDA tensor [batch][rows][heads][head dim] of fp32 or bf16 is wanted");
  const int dev = current(t, "x");
  const int64_t d = t.size(3);
  const Rows in(x[0], "x", -1, d, t.scalar_type(), dev);
  const int32_t* positions = ints<int32_t>(x[1], {in.batch, in.rows}, "positions", dev);
  const Frequencies freq(x[2], dev);
  const int interleaved = truth(x[4]);
  const double magnitude = real(x[5]);
  Tensor made;
  void* out;
  int64_t ld_out = (int64_t)in.heads * d;
  if (x[3] == Py_None) {
    made = fresh(t.sizes(), t.scalar_type(), dev);
    out = made.data_ptr();
  } else {
    const Rows to(x[3], "out", in.heads, d, t.scalar_type(), dev);
    if (to.batch != in.batch || to.rows != in.rows) wrong(tensor(x[3], "out"), t.scalar_type(), t.sizes(), "out", dev);
    out = to.at;
    ld_out = to.ld;
  }
  const int head_dim = small(d);
  call("poss_rotary", dev, [&](poss_stream stream) {
    return poss_rotary(in.at, in.ld, out, ld_out, t.scalar_type() == at::kBFloat16 ? POSS_BF16 : POSS_FP32, (int64_t)in.batch * in.rows,
                       in.heads, head_dim, positions, freq.at, freq.rot_dim, interleaved, (float)magnitude, stream);
  });
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[3]);
  return x[3];
}

// k, v, kv_pages, layer, tables, prefix_len, freq, positions, q, out_q, interleaved, magnitude, n_rows, status
POSS_CALL(append_rotary, 14) {
  const Pool pool(x[2]);
  const int dev = pool.dev;
  const Rows k(x[0], "k", pool.p.n_kv_heads, pool), v(x[1], "v", pool.p.n_kv_heads, pool);
  if (v.ld != k.ld || v.batch != k.batch || v.rows != k.rows) refuse("k and v: the same shape and the same strides are wanted");
  const Table t(x[4], "tables", dev);
  if (t.n != k.batch) wrong(tensor(x[4], "tables"), at::kInt, {k.batch, t.max_pages}, "tables", dev);
  const int layer = integer(x[3]);
  const int32_t* prefix = ints<int32_t>(x[5], {k.batch}, "prefix_len", dev);
  const Frequencies freq(x[6], dev);
  const int32_t* positions = opt_ints(x[7], {k.batch, k.rows}, "positions", dev);
  const int interleaved = truth(x[10]);
  const double magnitude = real(x[11]);
  const int32_t* n_rows = opt_ints(x[12], {k.batch}, "n_rows", dev);
  int32_t* status = opt_ints(x[13], {1}, "status", dev);
  const void* q = nullptr;
  void* out = nullptr;
  int64_t ld_q = 0, ld_out = 0;
  int heads = 0;
  Tensor made;
  if (x[8] != Py_None) {
    const Rows in(x[8], "q", -1, pool);
    if (in.batch != k.batch || in.rows != k.rows)
      wrong(tensor(x[8], "q"), pool.type, {k.batch, k.rows, in.heads, pool.p.head_dim}, "q", dev);
    q = in.at;
    ld_q = in.ld;
    heads = in.heads;
    ld_out = (int64_t)heads * pool.p.head_dim;
    if (x[9] == Py_None) {
      made = fresh(tensor(x[8], "q").sizes(), pool.type, dev);
      out = made.data_ptr();
    } else {
      const Rows to(x[9], "out_q", heads, pool);
      if (to.batch != k.batch || to.rows != k.rows)
        wrong(tensor(x[9], "out_q"), pool.type, {k.batch, k.rows, heads, pool.p.head_dim}, "out_q", dev);
      out = to.at;
      ld_out = to.ld;
    }
  } else if (x[9] != Py_None) {
    refuse("out_q: there are no queries");
  }
  call("poss_pages_append_rotary", dev, [&](poss_stream stream) {
    return poss_pages_append_rotary(&pool.p, layer, pool.pages, t.at, t.max_pages, k.batch, k.rows, k.at, v.at, k.ld, heads, q, ld_q, out,
                                    ld_out, prefix, n_rows, positions, freq.at, freq.rot_dim, interleaved, (float)magnitude, status,
                                    stream);
  });
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[9]);
  return x[9];
}

// q, kv_pages, mass, layer, tables, prefix_len, anc_mask, scale, n_rows, row_weights, out, workspace, status
POSS_CALL(attention_mass, 13) {
  const Pool pool(x[1]);
  const int dev = pool.dev;
  const Rows q(x[0], "q", -1, pool);
  const int b = q.batch, r = q.rows;
  const Mass mass(x[2], "mass", pool, b);
  const int64_t shape[4] = {b, r, q.heads, pool.p.head_dim};
  const double scale = real(x[7]);
  Tensor made;
  void* out;
  if (x[10] == Py_None) {
    made = fresh(shape, pool.type, dev);
    out = made.data_ptr();
  } else {
    out = arg(x[10], pool.type, shape, "out", dev);
  }
  if (b && r) {
    const Table t(x[4], "tables", dev);
    if (t.n != b) wrong(tensor(x[4], "tables"), at::kInt, {b, t.max_pages}, "tables", dev);
    const int layer = integer(x[3]);
    const int32_t* prefix = ints<int32_t>(x[5], {b}, "prefix_len", dev);
    const int32_t* n_rows = opt_ints(x[8], {b}, "n_rows", dev);
    const int64_t* mask = ints<int64_t>(x[6], {b, r, (r + 63) / 64}, "anc_mask", dev);
    const float* weights = static_cast<const float*>(opt(x[9], at::kFloat, {b, r}, "row_weights", dev));
    int32_t* status = opt_ints(x[12], {1}, "status", dev);
    const Scratch ws(x[11], poss_paged_attention_mass_workspace_bytes(&pool.p, b, r, q.heads, t.max_pages), dev);
    call("poss_paged_tree_attention_mass", dev, [&](poss_stream stream) {
      return poss_paged_tree_attention_mass(&pool.p, layer, pool.pages, mass.at, mass.slots, t.at, t.max_pages, b, r, q.heads, q.at, q.ld,
                                            prefix, n_rows, reinterpret_cast<const uint64_t*>(mask), weights, (float)scale, out, ws.at,
                                            ws.bytes, status, stream);
    });
  }
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[10]);
  return x[10];
}

POSS_CALL(evict, 12) {  // kv_pages, mass, tables, seq_len, keep, first, recent, out_mass, out_len, workspace, status, refs
  const Pool pool(x[0]);
  const int dev = pool.dev;
  const Table t(x[2], "tables", dev);
  const int b = t.n;
  const Mass mass(x[1], "mass", pool, b), out_mass(x[7] == Py_None ? x[1] : x[7], "out_mass", pool, b);
  if (out_mass.slots != mass.slots) refuse("out_mass: the shape of mass is wanted");
  const int32_t* len = ints<int32_t>(x[3], {b}, "seq_len", dev);
  const int32_t* keep = ints<int32_t>(x[4], {b}, "keep", dev);
  const int first = integer(x[5]), recent = integer(x[6]);
  int32_t* status = opt_ints(x[10], {1}, "status", dev);
  Tensor made;
  int32_t* out;
  if (x[8] == Py_None) {
    made = fresh({b}, at::kInt, dev);
    out = static_cast<int32_t*>(made.data_ptr());
  } else {
    out = ints<int32_t>(x[8], {b}, "out_len", dev);
  }
  const int32_t* refs = opt_ints(x[11], {pool.p.n_pages}, "refs", dev);
  const Scratch ws(x[9], poss_pages_evict_workspace_bytes(&pool.p, b, t.max_pages), dev);
  call("poss_pages_evict", dev, [&](poss_stream stream) {
    return poss_pages_evict_refs(&pool.p, pool.pages, t.at, t.max_pages, b, refs, mass.at, out_mass.at, mass.slots, len, keep, first, recent,
                                 out, ws.at, ws.bytes, status, stream);
  });
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(x[8]);
  return x[8];
}

POSS_CALL(token_logprobs, 6) {  // logits, tokens, token_rows, topk, temperature, out
  const Tensor& logits = tensor(x[0], "logits");
  if (logits.dim() != 2 || !pool_type(logits.scalar_type())) refuse("logits: a CUDA tensor [rows][vocab] of fp32 or bf16 is wanted");
  const int dev = current(logits, "logits");
  const int rows = small(logits.size(0)), vocab = small(logits.size(1));
  const int64_t ld = rows > 1 ? logits.stride(0) : vocab;
  if ((vocab > 1 && logits.stride(1) != 1) || ld < vocab)
    refuse("logits: rows of consecutive elements that do not overlap are wanted, got strides " + list(logits.strides()));
  int n = 0;
  if (x[1] != Py_None) {
    const Tensor& t = tensor(x[1], "tokens");
    if (t.dim() != 1) refuse("tokens: a tensor of one dimension is wanted");
    n = small(t.size(0));
  }
  const int32_t* tokens = opt_ints(x[1], {n}, "tokens", dev);
  const int32_t* token_rows = opt_ints(x[2], {n}, "token_rows", dev);
  const int k = integer(x[3]);
  const double temperature = real(x[4]);
  if (k < 0 || k > POSS_MAX_TOPK) refuse("topk: 0 to " + std::to_string(POSS_MAX_TOPK) + " are wanted, got " + std::to_string(k));
  Outputs out(x[5]);
  float* logp = static_cast<float*>(out.get("logp", at::kFloat, {n}, "out logp", dev));
  float* lse = static_cast<float*>(out.get("lse", at::kFloat, {rows}, "out lse", dev));
  float* entropy = static_cast<float*>(out.get("entropy", at::kFloat, {rows}, "out entropy", dev));
  int32_t* top = static_cast<int32_t*>(out.get("top_tokens", at::kInt, {rows, k}, "out top_tokens", dev));
  float* top_logp = static_cast<float*>(out.get("top_logp", at::kFloat, {rows, k}, "out top_logp", dev));
  call("poss_token_logprobs", dev, [&](poss_stream stream) {
    return poss_token_logprobs(logits.data_ptr(), ld, logits.scalar_type() == at::kBFloat16 ? POSS_BF16 : POSS_FP32, rows, vocab,
                               (float)temperature, tokens, token_rows, n, logp, lse, entropy, k, top, top_logp, stream);
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
                         {"rotary", FAST(rotary)},           {"append_rotary", FAST(append_rotary)},
                         {"attention_mass", FAST(attention_mass)}, {"evict", FAST(evict)},
                         {"token_logprobs", FAST(token_logprobs)},
                         {"bind", bind, METH_O, nullptr},    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_calls() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_with_torch", POSS_BUILT_WITH_TORCH)) Py_CLEAR(m);
  return m;
}
