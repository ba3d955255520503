// The operators between the layers, from Python tensors to the C functions without ctypes: a module of the
// package. Every function takes the usual call (tensors on the current device, of the expected shapes and
// types, on the current stream), makes it and returns its status; anything else it leaves alone and returns
// None, and the binding in Python, which has every check and message, takes the call.
//
// A decode step makes a few of these calls per layer, and its kernels take as little as 2 us: a norm's call
// costs the host 2.8 us so, 2.5 of them the launch, and 5.7 by way of ctypes.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "aqmb.h"

namespace {

using at::ScalarType;
using at::Tensor;

// The library's functions, at the addresses where the binding loaded them.
decltype(&aqmb_rms_norm) f_norm;
decltype(&aqmb_w4_gemv) f_w4;
decltype(&aqmb_paged_attention) f_attention;
decltype(&aqmb_paged_attention_workspace_bytes) f_workspace;
decltype(&aqmb_kv_append) f_append;
decltype(&aqmb_kv_copy_pages) f_copy;
decltype(&aqmb_rotary) f_rotary;
decltype(&aqmb_rotary_append) f_rotary_append;
decltype(&aqmb_adapters_add) f_adapters;
decltype(&aqmb_adapters_workspace_bytes) f_adapters_workspace;
decltype(&aqmb_log_probs) f_log_probs;
decltype(&aqmb_log_probs_workspace_bytes) f_log_probs_workspace;

struct NotUsual {};
void need(bool usual) {
  if (!usual) throw NotUsual{};
}

aqmb_dtype dtype_of(const Tensor& t) {
  switch (t.scalar_type()) {
    case ScalarType::Half: return AQMB_F16;
    case ScalarType::BFloat16: return AQMB_BF16;
    case ScalarType::Float: return AQMB_F32;
    case ScalarType::Float8_e4m3fn: return AQMB_F8;
    case ScalarType::Char: return AQMB_I8;
    default: throw NotUsual{};
  }
}

// A torch.Tensor or Parameter on device dev (-1: on any GPU) that is not empty, unless it may be.
const Tensor& tensor(PyObject* o, int dev, bool may_be_empty = false) {
  need(THPVariable_CheckExact(o));
  const Tensor& t = THPVariable_Unpack(o);
  need(t.is_cuda() && (may_be_empty || t.numel() > 0) && (dev < 0 || t.get_device() == dev));
  return t;
}
int current(const Tensor& t) {
  const int dev = t.get_device();
  need(c10::hip::current_device() == dev);
  return dev;
}
void* dense(PyObject* o, int dev, ScalarType type, int64_t n) {
  const Tensor& t = tensor(o, dev);
  need(t.scalar_type() == type && t.numel() == n && t.is_contiguous());
  return t.data_ptr();
}
// The stride between the rows of a tensor [rows][cols] whose rows are dense.
int64_t rows_of(const Tensor& t, int64_t rows, int64_t cols) {
  need(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && (t.stride(1) == 1 || cols == 1));
  return rows > 1 ? t.stride(0) : cols;
}
// The same of a tensor [rows][heads][dim].
int64_t rows_of(const Tensor& t, int64_t rows, int64_t heads, int64_t dim) {
  need(t.dim() == 3 && t.size(0) == rows && t.size(1) == heads && t.size(2) == dim);
  need((t.stride(2) == 1 || dim == 1) && (t.stride(1) == dim || heads == 1));
  return rows > 1 ? t.stride(0) : heads * dim;
}
int whole(int64_t n) {
  need(n >= 0 && n <= INT_MAX);
  return (int)n;
}
int64_t integer(PyObject* o) {
  need(PyLong_Check(o));
  int over = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &over);
  need(!over);
  return v;
}
float real(PyObject* o) {
  need(PyFloat_Check(o));
  return (float)PyFloat_AS_DOUBLE(o);
}
template <class T>
T address(PyObject* o) {
  need(PyLong_Check(o));
  void* p = PyLong_AsVoidPtr(o);
  need(p != nullptr);
  return static_cast<T>(p);
}
aqmb_stream_t stream(int dev) { return (aqmb_stream_t)c10::hip::getCurrentHIPStream(dev).stream(); }

// body() makes the call and returns its status. Nothing it throws passes into Python.
template <class F>
PyObject* usual(F body) {
  try {
    return PyLong_FromLong(body());
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}
// A launch may wait for room in the queue: not with the interpreter's lock.
template <class F>
int launch(F call) {
  int s;
  Py_BEGIN_ALLOW_THREADS;
  s = call();
  Py_END_ALLOW_THREADS;
  return s;
}

// The caller's workspace, or `bytes` bytes beside `like` from the allocator, which ties them to the current stream.
struct Workspace {
  Tensor own;
  void* data = nullptr;
  size_t bytes;
  Workspace(PyObject* given, size_t needed, const Tensor& like, int dev) : bytes(needed) {
    if (given != Py_None) {
      const Tensor& t = tensor(given, dev, true);
      need(t.is_contiguous());        // its bytes are its own
      data = t.data_ptr();
      bytes = (size_t)t.numel() * t.element_size();
    } else if (needed) {
      own = at::empty({(int64_t)needed}, like.options().dtype(ScalarType::Byte));
      data = own.data_ptr();
    }
  }
};

// (x, weight, y, eps, weight_offset, residual, residual_out, scales, scale_group)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return usual([&] {
    need(n == 9);
    const Tensor& x = tensor(a[0], -1);
    const int dev = current(x);
    const Tensor& y = tensor(a[2], dev);
    need(x.dim() == 2);
    const int rows = whole(x.size(0)), cols = whole(x.size(1));
    const aqmb_dtype dt = dtype_of(x), ydt = dtype_of(y);
    const int64_t xs = rows_of(x, rows, cols), ys = rows_of(y, rows, cols);
    const void* w = dense(a[1], dev, x.scalar_type(), cols);
    const float eps = real(a[3]), w0 = real(a[4]);
    const void* r = nullptr;
    void* ro = nullptr;
    int64_t rs = 0;
    if (a[5] != Py_None || a[6] != Py_None) {
      const Tensor &in = tensor(a[5], dev), &out = tensor(a[6], dev);
      need(in.scalar_type() == x.scalar_type() && out.scalar_type() == x.scalar_type());
      rs = rows_of(in, rows, cols);
      need(rows_of(out, rows, cols) == rs);
      r = in.data_ptr();
      ro = out.data_ptr();
    }
    float* scales = nullptr;
    const int group = whole(integer(a[8]));
    if (a[7] != Py_None)
      scales = (float*)dense(a[7], dev, ScalarType::Float, (int64_t)rows * (group ? (cols - 1) / group + 1 : 1));
    const void* xp = x.data_ptr();
    void* yp = y.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_norm(xp, dt, xs, r, ro, rs, w, w0, eps, rows, cols, yp, ydt, ys, scales, group, st); });
  });
}

// (layer, d_out, d_in, group_size, x, y, x_scales)
PyObject* w4_gemv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return usual([&] {
    need(n == 7);
    const aqmb_w4_t layer = address<aqmb_w4_t>(a[0]);
    const int64_t d_out = integer(a[1]), d_in = integer(a[2]), size = integer(a[3]);
    const Tensor& x = tensor(a[4], -1);
    const int dev = current(x);
    const Tensor& y = tensor(a[5], dev);
    need(x.dim() == 2);
    const int batch = whole(x.size(0));
    const aqmb_dtype dt = dtype_of(x), ydt = dtype_of(y);
    const int64_t xs = rows_of(x, batch, d_in), ys = rows_of(y, batch, d_out);
    const float* scales = nullptr;
    int group = 0;
    if (a[6] != Py_None) {            // one scale per row, or one per group
      if (tensor(a[6], dev).numel() != batch) group = whole(size);
      scales = (const float*)dense(a[6], dev, ScalarType::Float, batch * (group ? (d_in - 1) / group + 1 : 1));
    }
    const void* xp = x.data_ptr();
    void* yp = y.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_w4(layer, xp, dt, xs, scales, group, batch, yp, ydt, ys, st); });
  });
}

// (descriptor, its device, q, page_table, lengths, out, scale, max_length, window, lse, workspace)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 11);
    const aqmb_kv_cache* c = address<const aqmb_kv_cache*>(a[0]);
    const Tensor& q = tensor(a[2], -1);
    const int dev = current(q);
    need(integer(a[1]) == dev);
    const Tensor &table = tensor(a[3], dev), &out = tensor(a[5], dev);
    need(q.dim() == 3 && out.scalar_type() == q.scalar_type());
    const int n = whole(q.size(0)), heads = whole(q.size(1));
    const aqmb_dtype dt = dtype_of(q);
    const int64_t qs = rows_of(q, n, heads, c->head_dim), os = rows_of(out, n, heads, c->head_dim);
    need(table.dim() == 2 && table.scalar_type() == ScalarType::Int);
    const int64_t per = table.size(1), ts = rows_of(table, n, per), most = per * c->page_size;
    const int32_t* lengths = (const int32_t*)dense(a[4], dev, ScalarType::Int, n);
    const float scale = real(a[6]);
    const int max_length = whole(a[7] == Py_None ? (most < 1 << 27 ? most : 1 << 27) : integer(a[7]));
    need(max_length <= most);
    const int window = whole(integer(a[8]));
    float* lse = a[9] == Py_None ? nullptr : (float*)dense(a[9], dev, ScalarType::Float, (int64_t)n * heads);
    size_t bytes = 0;
    need(f_workspace(c, heads, n, max_length, window, &bytes) == AQMB_OK);
    const Workspace work(a[10], bytes, q, dev);
    const void* qp = q.data_ptr();
    void* op = out.data_ptr();
    const int32_t* tp = (const int32_t*)table.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] {
      return f_attention(c, qp, dt, qs, heads, tp, ts, lengths, n, max_length, scale, window, op, os, lse, work.data, work.bytes, st);
    });
  });
}

// (descriptor, its device, k, v, slots)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 5);
    const aqmb_kv_cache* c = address<const aqmb_kv_cache*>(a[0]);
    const Tensor& k = tensor(a[2], -1);
    const int dev = current(k);
    need(integer(a[1]) == dev);
    const Tensor& v = tensor(a[3], dev);
    need(k.dim() == 3 && v.scalar_type() == k.scalar_type());
    const int n = whole(k.size(0));
    const aqmb_dtype dt = dtype_of(k);
    const int64_t ks = rows_of(k, n, c->n_kv_heads, c->head_dim), vs = rows_of(v, n, c->n_kv_heads, c->head_dim);
    const int64_t* slots = (const int64_t*)dense(a[4], dev, ScalarType::Long, n);
    const void *kp = k.data_ptr(), *vp = v.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_append(c, kp, ks, vp, vs, dt, slots, n, st); });
  });
}

// (descriptor, its device, q, positions, q_out, k, k_out)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 7);
    const aqmb_rotary_desc* r = address<const aqmb_rotary_desc*>(a[0]);
    const Tensor& q = tensor(a[2], -1);
    const int dev = current(q);
    need(integer(a[1]) == dev);
    const Tensor& out = tensor(a[4], dev);
    need(q.dim() == 3 && out.scalar_type() == q.scalar_type());
    const int n = whole(q.size(0)), heads = whole(q.size(1)), dim = whole(q.size(2));
    const aqmb_dtype dt = dtype_of(q);
    const int64_t qs = rows_of(q, n, heads, dim), os = rows_of(out, n, heads, dim);
    const int64_t* positions = (const int64_t*)dense(a[3], dev, ScalarType::Long, n);
    const void* kp = nullptr;
    void* kop = nullptr;
    int64_t ks = 0, kos = 0;
    int kv = 0;
    if (a[5] != Py_None || a[6] != Py_None) {
      const Tensor &k = tensor(a[5], dev), &ko = tensor(a[6], dev);
      need(k.dim() == 3 && k.scalar_type() == q.scalar_type() && ko.scalar_type() == q.scalar_type());
      kv = whole(k.size(1));
      ks = rows_of(k, n, kv, dim);
      kos = rows_of(ko, n, kv, dim);
      kp = k.data_ptr();
      kop = ko.data_ptr();
    }
    const void* qp = q.data_ptr();
    void* op = out.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_rotary(r, qp, qs, op, os, heads, kp, ks, kop, kos, kv, dt, dim, positions, n, st); });
  });
}

// (cache's descriptor, its device, rotary's descriptor, its device, q, k, v, positions, slots, q_out)
PyObject* rotary_append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 10);
    const aqmb_kv_cache* c = address<const aqmb_kv_cache*>(a[0]);
    const aqmb_rotary_desc* r = address<const aqmb_rotary_desc*>(a[2]);
    const Tensor& q = tensor(a[4], -1);
    const int dev = current(q);
    need(integer(a[1]) == dev && integer(a[3]) == dev);
    const Tensor &k = tensor(a[5], dev), &v = tensor(a[6], dev), &out = tensor(a[9], dev);
    need(q.dim() == 3 && out.scalar_type() == q.scalar_type() && k.scalar_type() == q.scalar_type() &&
         v.scalar_type() == q.scalar_type());
    const int n = whole(q.size(0)), heads = whole(q.size(1));
    const aqmb_dtype dt = dtype_of(q);
    const int64_t qs = rows_of(q, n, heads, c->head_dim), os = rows_of(out, n, heads, c->head_dim);
    const int64_t ks = rows_of(k, n, c->n_kv_heads, c->head_dim), vs = rows_of(v, n, c->n_kv_heads, c->head_dim);
    const int64_t* positions = (const int64_t*)dense(a[7], dev, ScalarType::Long, n);
    const int64_t* slots = (const int64_t*)dense(a[8], dev, ScalarType::Long, n);
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    void* op = out.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_rotary_append(c, r, qp, qs, op, os, heads, kp, ks, vp, vs, dt, positions, slots, n, st); });
  });
}

// (descriptor, its device, x, index, base, out, workspace)
PyObject* adapters_add(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 7);
    const aqmb_adapters* ad = address<const aqmb_adapters*>(a[0]);
    const Tensor& x = tensor(a[2], -1);
    const int dev = current(x);
    need(integer(a[1]) == dev && x.dim() == 2 && dtype_of(x) == ad->dtype);
    const Tensor &base = tensor(a[4], dev), &out = tensor(a[5], dev);
    need(out.scalar_type() == base.scalar_type());
    const int n = whole(x.size(0));
    const aqmb_dtype dt = dtype_of(base);
    const int64_t xs = rows_of(x, n, ad->d_in), bs = rows_of(base, n, ad->d_out), os = rows_of(out, n, ad->d_out);
    const int32_t* index = (const int32_t*)dense(a[3], dev, ScalarType::Int, n);
    size_t bytes = 0;
    need(f_adapters_workspace(ad, n, &bytes) == AQMB_OK);
    const Workspace work(a[6], bytes, x, dev);
    const void *xp = x.data_ptr(), *bp = base.data_ptr();
    void* op = out.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_adapters(ad, xp, xs, index, n, bp, bs, op, os, dt, work.data, work.bytes, st); });
  });
}

// (logits, targets, logprobs, scale, lse, entropy, top_ids, top_logprobs, workspace)
PyObject* log_probs(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 9);
    const Tensor& z = tensor(a[0], -1);
    const int dev = current(z);
    need(z.dim() == 2);
    const int rows = whole(z.size(0)), vocab = whole(z.size(1));
    const aqmb_dtype dt = dtype_of(z);
    const int64_t stride = rows_of(z, rows, vocab);
    const float scale = real(a[3]);
    // Columns of a dense tensor [rows][n] or [rows], of at least one value.
    const auto columns = [&](PyObject* o, ScalarType type, void** data) {
      const Tensor& t = tensor(o, dev);
      need((t.dim() == 1 || t.dim() == 2) && t.size(0) == rows && t.scalar_type() == type && t.is_contiguous());
      *data = t.data_ptr();
      return whole(t.numel() / rows);
    };
    void *targets = nullptr, *lp = nullptr, *ids = nullptr, *tops = nullptr;
    int n = 0, top = 0;
    if (a[1] != Py_None || a[2] != Py_None) {
      n = columns(a[1], ScalarType::Long, &targets);
      lp = dense(a[2], dev, ScalarType::Float, (int64_t)rows * n);
    }
    float* lse = a[4] == Py_None ? nullptr : (float*)dense(a[4], dev, ScalarType::Float, rows);
    float* entropy = a[5] == Py_None ? nullptr : (float*)dense(a[5], dev, ScalarType::Float, rows);
    if (a[6] != Py_None) top = columns(a[6], ScalarType::Long, &ids);
    if (a[7] != Py_None) {
      const int k = columns(a[7], ScalarType::Float, &tops);
      need(top == 0 || k == top);
      top = k;
    }
    size_t bytes = 0;
    need(f_log_probs_workspace(dt, rows, vocab, top, &bytes) == AQMB_OK);
    const Workspace work(a[8], bytes, z, dev);
    const void* zp = z.data_ptr();
    const aqmb_stream_t st = stream(dev);
    return launch([&] {
      return f_log_probs(zp, dt, stride, rows, vocab, scale, (const int64_t*)targets, n, (float*)lp, lse, entropy,
                         (int64_t*)ids, (float*)tops, top, work.data, work.bytes, st);
    });
  });
}

PyObject *s_address, *s_device;       // names of two attributes of KVCache

int64_t attribute(PyObject* o, PyObject* name) {
  PyObject* v = PyObject_GetAttr(o, name);
  need(v != nullptr);
  const int64_t n = PyLong_AsLongLong(v);
  Py_DECREF(v);
  need(!PyErr_Occurred());
  return n;
}

// (list or tuple of KVCache, src, dst)
PyObject* kv_copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return usual([&] {
    need(n_args == 3 && (PyList_Check(a[0]) || PyTuple_Check(a[0])));
    const Py_ssize_t caches = PySequence_Fast_GET_SIZE(a[0]);
    need(caches >= 1 && caches <= AQMB_MAX_CACHES);
    const Tensor& src = tensor(a[1], -1);
    const int dev = current(src);
    const int64_t n = src.numel();
    aqmb_kv_cache c[AQMB_MAX_CACHES];
    for (Py_ssize_t i = 0; i < caches; ++i) {
      PyObject* cache = PySequence_Fast_GET_ITEM(a[0], i);
      need(attribute(cache, s_device) == dev);
      const auto* desc = reinterpret_cast<const aqmb_kv_cache*>(attribute(cache, s_address));
      need(desc != nullptr);
      c[i] = *desc;
    }
    const int32_t *s = (const int32_t*)dense(a[1], dev, ScalarType::Int, n), *d = (const int32_t*)dense(a[2], dev, ScalarType::Int, n);
    const int pairs = whole(n);
    const aqmb_stream_t st = stream(dev);
    return launch([&] { return f_copy(c, (int)caches, s, d, pairs, st); });
  });
}

// (rms_norm, w4_gemv, paged_attention, its workspace_bytes, kv_append, kv_copy_pages): the functions' addresses.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[6];
  if (n != 6) return PyErr_Format(PyExc_TypeError, "bind takes six addresses");
  for (int i = 0; i < 6; ++i)
    if (!(f[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "a null address");
  f_norm = (decltype(f_norm))f[0];
  f_w4 = (decltype(f_w4))f[1];
  f_attention = (decltype(f_attention))f[2];
  f_workspace = (decltype(f_workspace))f[3];
  f_append = (decltype(f_append))f[4];
  f_copy = (decltype(f_copy))f[5];
  Py_RETURN_NONE;
}

// (rotary, rotary_append, adapters_add, its workspace_bytes, log_probs, its workspace_bytes): the functions' addresses.
PyObject* bind_requests(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[6];
  if (n != 6) return PyErr_Format(PyExc_TypeError, "bind_requests takes six addresses");
  for (int i = 0; i < 6; ++i)
    if (!(f[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "a null address");
  f_rotary = (decltype(f_rotary))f[0];
  f_rotary_append = (decltype(f_rotary_append))f[1];
  f_adapters = (decltype(f_adapters))f[2];
  f_adapters_workspace = (decltype(f_adapters_workspace))f[3];
  f_log_probs = (decltype(f_log_probs))f[4];
  f_log_probs_workspace = (decltype(f_log_probs_workspace))f[5];
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(rms_norm), METHOD(w4_gemv), METHOD(paged_attention),
                         METHOD(kv_append), METHOD(kv_copy_pages), METHOD(bind_requests), METHOD(rotary),
                         METHOD(rotary_append), METHOD(adapters_add), METHOD(log_probs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_direct", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__direct() {
  s_address = PyUnicode_InternFromString("_address");
  s_device = PyUnicode_InternFromString("device_index");
  return s_address && s_device ? PyModule_Create(&module) : nullptr;
}
