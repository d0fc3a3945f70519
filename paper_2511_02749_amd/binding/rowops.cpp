// The row operators on torch tensors (row_ops.py): types, shapes and devices are checked here,
// sizes, strides and alignment by the library, whose entries bind() is given.
//
// Native, since a call reads the attributes of up to a dozen tensors, which takes longer from
// Python than the launches: one row of head norms 8.8 -> 4.0 us, of adapters 12.0 -> 8.0.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <array>
#include <exception>
#include <map>
#include <string>

#include "spanq.h"

namespace {

struct Bad {  // an argument to refuse
  std::string what;
};
struct Raised {};  // a Python error is set

// what bind() is given, kept for the life of the process
struct {
  decltype(&span_qk_norm_rope) qk_norm_rope;
  decltype(&span_adapter_workspace) adapter_workspace;
  decltype(&span_adapter_apply) adapter_apply;
  decltype(&span_verify_workspace) verify_workspace;
  decltype(&span_verify_drafts) verify_drafts;
  PyObject *error, *check, *raw_stream, *scratch;
} bound;

// A new reference, or a Python error passed on.
struct Ref {
  PyObject* p;
  explicit Ref(PyObject* o) : p(o) {
    if (!p) throw Raised{};
  }
  Ref(Ref&& o) : p(o.p) { o.p = nullptr; }
  Ref(const Ref&) = delete;
  ~Ref() { Py_XDECREF(p); }
};

std::string list_of(at::IntArrayRef v) {
  std::string s = "(";
  for (const int64_t i : v) s += std::to_string(i) + ", ";
  return s + ")";
}

std::string said(const at::Tensor& t) {
  return std::string(c10::toString(t.scalar_type())) + " " + list_of(t.sizes()) + " on " + t.device().str();
}

// The tensor of an argument, null for None.
const at::Tensor* tensor(const char* name, PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Bad{std::string(name) + " must be a tensor"};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || t.is_neg()) throw Bad{std::string(name) + " must be a plain strided tensor"};
  return &t;
}
const at::Tensor& needed(const char* name, PyObject* o) {
  const at::Tensor* t = tensor(name, o);
  if (!t) throw Bad{std::string(name) + " is needed"};
  return *t;
}

bool lies_on(const at::Tensor& t, int gpu) { return t.is_cuda() && t.get_device() == gpu; }

int gpu_of(const char* name, const at::Tensor* t) {
  if (!t || !t->is_cuda()) throw Bad{std::string(name) + " must be a tensor on a GPU"};
  return static_cast<int>(t->get_device());
}

void* address(const at::Tensor& t) { return const_cast<void*>(t.const_data_ptr()); }

// A tensor that a call has written: what autograd saved of it before is not what it holds now.
void written(const at::Tensor* t) {
  if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

struct Rows {
  void* at;
  int64_t stride;
};

// A [rows, width] or [rows, heads, dim] tensor of that shape whose rows are dense.
Rows rows_of(const char* name, const at::Tensor& t, at::ScalarType type, int gpu, at::IntArrayRef shape) {
  if (t.scalar_type() != type || !lies_on(t, gpu) || t.sizes() != shape)
    throw Bad{std::string(name) + " must be " + c10::toString(type) + " " + list_of(shape) + " on GPU " + std::to_string(gpu) +
              ", not " + said(t)};
  const int64_t width = shape.back(), row = shape.size() == 3 ? width * shape[1] : width;
  if (t.is_contiguous()) return {address(t), row};
  const at::IntArrayRef st = t.strides();
  if (st.back() != 1 && width > 1) throw Bad{std::string("the elements of a row of ") + name + " must follow one another"};
  if (shape.size() == 3 && st[1] != width && shape[1] > 1)
    throw Bad{std::string("the heads of a row of ") + name + " must follow one another"};
  // the stride of a single row says nothing
  return {address(t), shape[0] > 1 ? st[0] : std::max(st[0], row)};
}

// A dense tensor of n elements, null for None.
template <class T>
T* list(const char* name, PyObject* o, at::ScalarType type, int gpu, int64_t n) {
  const at::Tensor* t = tensor(name, o);
  if (!t) return nullptr;
  if (t->scalar_type() != type || !lies_on(*t, gpu) || t->numel() != n || !t->is_contiguous())
    throw Bad{std::string(name) + " must be contiguous, " + c10::toString(type) + " on GPU " + std::to_string(gpu) + ", with " +
              std::to_string(n) + " elements, not " + said(*t)};
  return static_cast<T*>(address(*t));
}

void* pointer(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}

// The stream of a call: an address, an object that has one, or None: the GPU's current one.
void* stream_of(PyObject* o, int gpu) {
  if (PyLong_Check(o)) return pointer(o);
  if (o != Py_None) {
    PyObject* of = PyObject_GetAttrString(o, "device_index");  // (not every object with a stream tells)
    if (!of) PyErr_Clear();
    const long index = of ? PyLong_AsLong(of) : gpu;
    Py_XDECREF(of);
    if (index == -1 && PyErr_Occurred()) throw Raised{};
    if (index != gpu) throw Bad{"the stream is GPU " + std::to_string(index) + "'s, the tensors lie on " + std::to_string(gpu)};
  }
  const Ref r(o == Py_None ? PyObject_CallFunction(bound.raw_stream, "i", gpu) : PyObject_GetAttrString(o, "cuda_stream"));
  return pointer(r.p);
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}

// A call's workspace: the caller's, or memory of the call's stream that goes back when the call has been
// enqueued.
struct Workspace {
  at::Tensor own;
  void* at = nullptr;
  size_t bytes = 0;

  Workspace(PyObject* given, int gpu, PyObject* stream, size_t need) {
    if (const at::Tensor* t = tensor("workspace", given)) {
      if (!lies_on(*t, gpu) || !t->is_contiguous())
        throw Bad{"workspace must be contiguous on GPU " + std::to_string(gpu)};
      own = *t;
    } else if (stream == Py_None) {
      own = at::empty({static_cast<int64_t>(need)},
                      at::TensorOptions().dtype(at::kByte).device(at::kCUDA, static_cast<c10::DeviceIndex>(gpu)));
    } else {
      const Ref r(PyObject_CallFunction(bound.scratch, "nOi", static_cast<Py_ssize_t>(need), stream, gpu));
      own = needed("workspace", r.p);
    }
    at = address(own);
    bytes = own.nbytes();
  }
};

void checked(int rc) {
  if (rc != SPAN_OK) Ref(PyObject_CallFunction(bound.check, "i", rc));  // raises
}

// A launch, with other threads let in.
template <class F>
void launch(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS rc = f();
  Py_END_ALLOW_THREADS checked(rc);
}

PyObject* refuse(const char* who, const std::string& what, int code = SPAN_EINVAL) {
  PyObject* e = PyObject_CallFunction(bound.error, "is", code, (std::string(who) + ": " + what).c_str());
  if (e) PyErr_SetObject(bound.error, e);
  Py_XDECREF(e);
  return nullptr;
}

template <class F>
PyObject* entry(const char* who, Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want || !bound.error) {
    PyErr_SetString(PyExc_TypeError, "arguments");
    return nullptr;
  }
  try {
    f();
    Py_RETURN_NONE;
  } catch (const Bad& b) {
    return refuse(who, b.what);
  } catch (const Raised&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    return refuse(who, e.what_without_backtrace(), SPAN_ENOMEM);
  } catch (const std::exception& e) {
    return refuse(who, e.what());
  }
}

// q, k, v, q_gain, k_gain, eps, q_out, k_out, v_out, rows, positions, rope_theta, stream
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return entry("qk_norm_rope", n_args, 13, [&] {
    static const char* const names[3] = {"q", "k", "v"};
    static const char* const outs[3] = {"q_out", "k_out", "v_out"};
    const at::Tensor *in[3], *out[3], *lead = nullptr;
    for (int i = 0; i < 3; ++i) {
      in[i] = tensor(names[i], a[i]);
      out[i] = tensor(outs[i], a[6 + i]);
      if (!in[i] != !out[i]) throw Bad{std::string(names[i]) + " and " + outs[i] + " go together"};
      if (!lead) lead = in[i];
    }
    const int gpu = gpu_of("q, k or v", lead);
    const at::ScalarType type = lead->scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || lead->dim() != 3)
      throw Bad{"rows must be bfloat16 or float32 [rows, heads, dim]"};
    const int64_t n = lead->size(0), dim = lead->size(2);
    int64_t out_rows = -1, heads[3] = {0, 0, 0};
    Rows from[3] = {}, to[3] = {};
    for (int i = 0; i < 3; ++i) {
      if (!in[i]) continue;
      heads[i] = in[i]->dim() == 3 ? in[i]->size(1) : lead->size(1);
      if (out_rows < 0) out_rows = out[i]->dim() ? out[i]->size(0) : 0;
      from[i] = rows_of(names[i], *in[i], type, gpu, {n, heads[i], dim});
      to[i] = rows_of(outs[i], *out[i], type, gpu, {out_rows, heads[i], dim});
    }
    if (in[1] && in[2] && heads[1] != heads[2]) throw Bad{"k and v must have the same heads"};
    span_qk_norm c{};
    c.q = from[0].at;
    c.k = from[1].at;
    c.v = from[2].at;
    c.q_out = to[0].at;
    c.k_out = to[1].at;
    c.v_out = to[2].at;
    c.q_gain = list<void>("q_gain", a[3], type, gpu, dim);
    c.k_gain = list<void>("k_gain", a[4], type, gpu, dim);
    c.rows = list<int32_t>("rows", a[9], at::kInt, gpu, n);
    c.positions = list<int32_t>("positions", a[10], at::kInt, gpu, n);
    c.q_stride = from[0].stride;
    c.k_stride = from[1].stride;
    c.v_stride = from[2].stride;
    c.q_out_stride = to[0].stride;
    c.k_out_stride = to[1].stride;
    c.v_out_stride = to[2].stride;
    c.n_rows = n;
    c.out_rows = out_rows;
    c.num_q_heads = static_cast<int32_t>(std::min<int64_t>(heads[0], INT32_MAX));
    c.num_kv_heads = static_cast<int32_t>(std::min<int64_t>(std::max(heads[1], heads[2]), INT32_MAX));
    c.head_dim = static_cast<int32_t>(std::min<int64_t>(dim, INT32_MAX));
    c.dtype = type == at::kBFloat16 ? SPAN_BF16 : SPAN_F32;
    c.device = gpu;
    c.eps = static_cast<float>(number(a[5]));
    c.rope_theta = static_cast<float>(number(a[11]));
    void* stream = stream_of(a[12], gpu);
    launch([&] { return bound.qk_norm_rope(&c, stream); });
    for (const at::Tensor* t : out) written(t);
  });
}

// The workspace of a call, from its sizes; told once for each.
size_t adapter_bytes(const span_adapter_call& c) {
  static std::map<std::array<int64_t, 8>, size_t> known;
  const std::array<int64_t, 8> key{c.n_rows, c.in_features, c.max_rank, c.n_parts, c.part_cols[0], c.part_cols[1],
                                   c.part_cols[2], c.part_cols[3]};
  const auto it = known.find(key);
  if (it != known.end()) return it->second;
  size_t bytes = 0;
  checked(bound.adapter_workspace(&c, &bytes));
  if (known.size() >= 1024) known.clear();
  known.emplace(key, bytes);
  return bytes;
}

// x, base, ids, a, b, scale, out, parts, ranks, workspace, stream
PyObject* adapter_apply(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return entry("adapter_apply", n_args, 11, [&] {
    const at::Tensor* x = tensor("x", a[0]);
    const int gpu = gpu_of("x", x);
    const at::Tensor &out = needed("out", a[6]), &wa = needed("a", a[3]), &wb = needed("b", a[4]);
    if (x->dim() != 2 || out.dim() != 2 || wa.dim() != 4) throw Bad{"x and out must have two dimensions, a four"};
    const int64_t n = x->size(0), width = x->size(1), cols = out.size(1), count = wa.size(0), rank = wa.size(2);
    int64_t parts[4] = {cols, 0, 0, 0}, n_parts = 1, sum = cols;
    if (a[7] != Py_None) {
      const Ref seq(PySequence_Fast(a[7], "parts must be a sequence"));
      n_parts = PySequence_Fast_GET_SIZE(seq.p);
      if (n_parts < 1 || n_parts > 4) throw Bad{"parts must be one to four column counts"};
      sum = 0;
      for (int64_t p = 0; p < n_parts; ++p) {
        parts[p] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq.p, p));
        if (parts[p] == -1 && PyErr_Occurred()) throw Raised{};
        if (parts[p] < 0 || parts[p] > cols) throw Bad{"parts must add up to out's columns"};
        sum += parts[p];
      }
    }
    if (wa.size(1) != n_parts || sum != cols || wa.size(3) != width || out.size(0) != n ||
        wb.sizes() != at::IntArrayRef({count, cols, rank}))
      throw Bad{"a must be [n, parts, rank, in], b [n, cols, rank], parts one to four column counts that add up to "
                "out's columns, out as many rows as x"};
    if (n > INT32_MAX || width > INT32_MAX || cols > INT32_MAX || count > INT32_MAX || rank > INT32_MAX)
      throw Bad{"sizes must be below 2^31"};
    const Rows rx = rows_of("x", *x, at::kBFloat16, gpu, {n, width});
    const Rows ro = rows_of("out", out, at::kBFloat16, gpu, {n, cols});
    const Rows rb = a[1] == a[6] ? ro : rows_of("base", needed("base", a[1]), at::kBFloat16, gpu, {n, cols});
    span_adapter_call c{};
    c.x = rx.at;
    c.base = rb.at;
    c.out = ro.at;
    c.ids = list<int32_t>("ids", a[2], at::kInt, gpu, n);
    c.a = list<void>("a", a[3], at::kBFloat16, gpu, wa.numel());
    c.b = list<void>("b", a[4], at::kBFloat16, gpu, wb.numel());
    c.scale = list<float>("scale", a[5], at::kFloat, gpu, count);
    c.ranks = list<int32_t>("ranks", a[8], at::kInt, gpu, count);
    c.x_stride = rx.stride;
    c.base_stride = rb.stride;
    c.out_stride = ro.stride;
    c.n_rows = n;
    c.in_features = static_cast<int32_t>(width);
    c.n_adapters = static_cast<int32_t>(count);
    c.max_rank = static_cast<int32_t>(rank);
    c.n_parts = static_cast<int32_t>(n_parts);
    for (int p = 0; p < 4; ++p) c.part_cols[p] = static_cast<int32_t>(parts[p]);
    c.device = gpu;
    void* stream = stream_of(a[10], gpu);
    const Workspace ws(a[9], gpu, a[10], a[9] == Py_None ? adapter_bytes(c) : 0);
    c.workspace = ws.at;
    c.workspace_bytes = ws.bytes;
    launch([&] { return bound.adapter_apply(&c, stream); });
    written(&out);
  });
}

// target_logits, drafts, u_accept, u_sample, temperature, accepted, tokens, draft_logits, n_drafts, row0,
// draft_row0, logprobs, workspace, stream
PyObject* verify_drafts(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return entry("verify_drafts", n_args, 14, [&] {
    const at::Tensor* target = tensor("target_logits", a[0]);
    const int gpu = gpu_of("target_logits", target);
    const at::Tensor& tokens = needed("tokens", a[6]);
    if (target->dim() != 2 || tokens.dim() != 2 || tokens.size(1) < 1)
      throw Bad{"target_logits must be [rows, vocab], tokens [requests, drafts + 1]"};
    const int64_t n = tokens.size(0), k = tokens.size(1) - 1, vocab = target->size(1);
    if (n > INT32_MAX || k > INT32_MAX || vocab > INT32_MAX) throw Bad{"sizes must be below 2^31"};
    const Rows rt = rows_of("target_logits", *target, at::kFloat, gpu, target->sizes());
    span_verify_call c{};
    // (a tensor of no rows may have no address, which would say that there is none: any other, never read)
    c.target_logits = static_cast<const float*>(rt.at ? rt.at : address(tokens));
    c.target_stride = rt.stride;
    c.target_rows = target->size(0);
    c.draft_stride = vocab;
    if (const at::Tensor* draft = tensor("draft_logits", a[7])) {
      if (draft->dim() != 2) throw Bad{"draft_logits must be [rows, vocab]"};
      const Rows rd = rows_of("draft_logits", *draft, at::kFloat, gpu, {draft->size(0), vocab});
      c.draft_logits = static_cast<const float*>(rd.at ? rd.at : address(tokens));
      c.draft_stride = rd.stride;
      c.draft_rows = draft->size(0);
    }
    c.drafts = list<int32_t>("drafts", a[1], at::kInt, gpu, n * k);
    c.u_accept = list<float>("u_accept", a[2], at::kFloat, gpu, n * k);
    c.u_sample = list<float>("u_sample", a[3], at::kFloat, gpu, n);
    c.temperature = list<float>("temperature", a[4], at::kFloat, gpu, n);
    c.accepted = list<int32_t>("accepted", a[5], at::kInt, gpu, n);
    c.tokens = list<int32_t>("tokens", a[6], at::kInt, gpu, n * (k + 1));
    c.n_drafts = list<int32_t>("n_drafts", a[8], at::kInt, gpu, n);
    c.target_row0 = list<int32_t>("row0", a[9], at::kInt, gpu, n);
    c.draft_row0 = list<int32_t>("draft_row0", a[10], at::kInt, gpu, n);
    c.logprobs = list<float>("logprobs", a[11], at::kFloat, gpu, n * (k + 1));
    c.n_requests = static_cast<int32_t>(n);
    c.max_drafts = static_cast<int32_t>(k);
    c.vocab = static_cast<int32_t>(vocab);
    c.device = gpu;
    if (k > 0 && (a[1] == Py_None || a[2] == Py_None)) throw Bad{"drafts need their tokens and random numbers"};
    if (a[3] == Py_None) throw Bad{"u_sample is needed"};
    void* stream = stream_of(a[13], gpu);
    size_t need = 0;
    if (a[12] == Py_None) checked(bound.verify_workspace(&c, &need));
    const Workspace ws(a[12], gpu, a[13], need);
    c.workspace = ws.at;
    c.workspace_bytes = ws.bytes;
    launch([&] { return bound.verify_drafts(&c, stream); });
    for (const int i : {5, 6, 11}) written(tensor("output", a[i]));
  });
}

// The library's five entries as addresses; SpanError; check(rc), which raises; the address of a GPU's current
// stream; scratch(bytes, stream, gpu), a tensor of memory of that stream.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 9) {
    PyErr_SetString(PyExc_TypeError, "bind takes nine arguments");
    return nullptr;
  }
  try {
    bound.qk_norm_rope = reinterpret_cast<decltype(bound.qk_norm_rope)>(pointer(a[0]));
    bound.adapter_workspace = reinterpret_cast<decltype(bound.adapter_workspace)>(pointer(a[1]));
    bound.adapter_apply = reinterpret_cast<decltype(bound.adapter_apply)>(pointer(a[2]));
    bound.verify_workspace = reinterpret_cast<decltype(bound.verify_workspace)>(pointer(a[3]));
    bound.verify_drafts = reinterpret_cast<decltype(bound.verify_drafts)>(pointer(a[4]));
  } catch (const Raised&) {
    return nullptr;
  }
  for (int i = 5; i < 9; ++i) Py_INCREF(a[i]);
  bound.error = a[5];
  bound.check = a[6];
  bound.raw_stream = a[7];
  bound.scratch = a[8];
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind>("bind"), method<qk_norm_rope>("qk_norm_rope"),
                         method<adapter_apply>("adapter_apply"), method<verify_drafts>("verify_drafts"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rowops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rowops() { return PyModule_Create(&module); }
