// The 4-bit cache's entries for Python: tensors are checked and turned into the C ABI's
// argument structures here.  A call through ctypes takes 7 to 8 us, most of it one
// attribute of a tensor after the other; the launch behind it takes 2.
//
// Every function takes its entry's address first (a ctypes function of the library that
// is loaded), checks its tensors, calls without the interpreter lock and returns the
// entry's code.  Faulty tensors raise ValueError, what is not a tensor TypeError.
#include <Python.h>

#include <c10/cuda/CUDAException.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "../../include/buddy.h"

namespace {

using at::ScalarType;

// What ends a call: the Python exception is set.
struct Failed {};

[[noreturn]] void wrong(const char* what, const char* wanted) {
  PyErr_Format(PyExc_ValueError, "%s: %s", what, wanted);
  throw Failed{};
}

const char* name_of(ScalarType t) {
  switch (t) {
    case ScalarType::Int: return "int32";
    case ScalarType::Long: return "int64";
    case ScalarType::Float: return "fp32";
    case ScalarType::Half: return "fp16";
    case ScalarType::BFloat16: return "bf16";
    case ScalarType::Byte: return "uint8";
    default: return "elements";
  }
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: a tensor is wanted", what);
    throw Failed{};
  }
  return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o, int64_t most = INT64_MAX) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed{};
  if (v > most || v < -most - 1) {
    PyErr_SetString(PyExc_OverflowError, "an argument does not fit in 32 bits");
    throw Failed{};
  }
  return v;
}
int32_t int32(PyObject* o) { return (int32_t)integer(o, INT32_MAX); }
int32_t int32(int64_t v, const char* what) {
  if (v > INT32_MAX) wrong(what, "fewer than 2^31 elements are wanted");
  return (int32_t)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Failed{};
  return (float)v;
}
// What a cache's address stands for: its argument, and the device of its pages.
struct Cache {
  buddy_kv4_cache c;
  int32_t device;
};

template <class F>
F entry(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no entry");
    throw Failed{};
  }
  return reinterpret_cast<F>(p);
}

// The device of a call: that of its first tensor.  The others are on it too.
struct Device {
  int index = -1;
  void take(const at::Tensor& t, const char* what) {
    if (index < 0) index = t.get_device();
    if (t.get_device() != index) wrong(what, "a tensor on the device of the others is wanted");
  }
};

const Cache* pages(Device& d, PyObject* address) {
  const Cache* const c = entry<const Cache*>(address);
  if (d.index < 0) d.index = c->device;
  if (d.index != c->device) wrong("pages", "a cache on the device of the tensors is wanted");
  return c;
}

// A contiguous CUDA tensor of n or more elements of a type.
const at::Tensor& vec(Device& d, PyObject* o, ScalarType type, int64_t n, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous() || t.numel() < n) {
    PyErr_Format(PyExc_ValueError, "%s: a contiguous CUDA tensor of %lld or more %s is wanted", what, (long long)n,
                 name_of(type));
    throw Failed{};
  }
  d.take(t, what);
  return t;
}
template <class T>
T* data(Device& d, PyObject* o, ScalarType type, int64_t n, const char* what) {
  return static_cast<T*>(vec(d, o, type, n, what).data_ptr());
}
template <class T>
T* data_or_null(Device& d, PyObject* o, ScalarType type, int64_t n, const char* what) {
  return o == Py_None ? nullptr : data<T>(d, o, type, n, what);
}

// [tokens, heads, head_dim] with whole heads one after the other: elements from token to token.
int64_t heads(Device& d, const at::Tensor& t, ScalarType type, int64_t tokens, int64_t n, int64_t hd, const char* what) {
  if (t.scalar_type() != type || !t.is_cuda() || t.dim() != 3 || t.size(0) != tokens || t.size(1) != n ||
      t.size(2) != hd || t.stride(2) != 1 || (t.stride(1) != hd && n > 1)) {
    PyErr_Format(PyExc_ValueError, "%s: CUDA %s (%lld, %lld, %lld) with whole heads one after the other is wanted", what,
                 name_of(type), (long long)tokens, (long long)n, (long long)hd);
    throw Failed{};
  }
  d.take(t, what);
  return t.stride(0);
}

// A rotary table: [positions, head_dim / 2].
const float* table(Device& d, PyObject* o, int64_t hd, const char* what, int32_t* positions) {
  const at::Tensor& t = vec(d, o, ScalarType::Float, 0, what);
  if (t.dim() != 2 || 2 * t.size(1) != hd) wrong(what, "[positions, head_dim / 2] is wanted");
  *positions = int32(t.size(0), what);
  return static_cast<const float*>(t.data_ptr());
}

int32_t dtype_of(ScalarType t) {
  return t == ScalarType::Float ? BUDDY_DTYPE_F32
         : t == ScalarType::BFloat16 ? BUDDY_DTYPE_BF16
         : t == ScalarType::Half ? BUDDY_DTYPE_F16 : -1;
}

// The stream given (a torch.cuda.Stream), or the current one of t's device.
void* stream_of(const at::Tensor& t, PyObject* stream) {
  if (stream == Py_None) return c10::cuda::getCurrentCUDAStream(t.get_device()).stream();
  PyObject* s = PyObject_GetAttrString(stream, "cuda_stream");
  if (!s) throw Failed{};
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (!p && PyErr_Occurred()) throw Failed{};
  return p;
}

// tensor, stream: the handle of the stream that a call with that tensor goes to.  For a cache
// that keeps a workspace for every stream: under a capture there is none to keep, since a
// replay may run next to calls that share the stream's.
PyObject* stream_for_workspace(PyObject* const* a) {
  const auto s = static_cast<cudaStream_t>(stream_of(tensor(a[0], "q"), a[1]));
  cudaStreamCaptureStatus status;
  C10_CUDA_CHECK(cudaStreamIsCapturing(s, &status));
  if (status != cudaStreamCaptureStatusNone) wrong("workspace", "a call that is captured in a graph wants one given");
  return PyLong_FromVoidPtr(s);
}

// The call, with its device as the current one.
template <class F>
PyObject* called(const Device& d, F&& f) {
  c10::cuda::OptionalCUDAGuard guard;
  if (c10::cuda::current_device() != d.index) guard.set_index((c10::DeviceIndex)d.index);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// A function of n arguments, with what it throws as Python exceptions.
template <int N, PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments are wanted", N);
    return nullptr;
  }
  try {
    return F(a);
  } catch (const Failed&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// entry, length, n_new, page_size, table, free_pages, free_head, kv_len, row_start, slot, pos,
// free_head_out, flags, stream
PyObject* page_plan(PyObject* const* a) {
  Device d;
  const at::Tensor& length = tensor(a[1], "length");
  const int64_t B = length.numel();
  const auto I = ScalarType::Int, L = ScalarType::Long;
  const at::Tensor& slot = vec(d, a[9], L, 0, "slot");
  const at::Tensor& table = vec(d, a[4], I, 0, "table");
  const at::Tensor& free = vec(d, a[5], I, 0, "free_pages");
  buddy_page_plan_args p{};
  p.batch = int32(B, "length");
  p.page_size = int32(a[3]);
  p.n_free = int32(free.numel(), "free_pages");
  p.n_tok = int32(slot.numel(), "slot");
  p.len = data<int32_t>(d, a[1], I, B, "length");
  p.n_new = data<int32_t>(d, a[2], I, B, "n_new");
  p.table = static_cast<int32_t*>(table.data_ptr());
  p.free_pages = static_cast<int32_t*>(free.data_ptr());
  p.free_head = data<int32_t>(d, a[6], I, 1, "free_head");
  p.kv_len = data<int32_t>(d, a[7], I, B, "kv_len");
  p.row_start = data<int32_t>(d, a[8], I, B + 1, "row_start");
  p.slot = static_cast<int64_t*>(slot.data_ptr());
  p.pos = data<int32_t>(d, a[10], I, p.n_tok, "pos");
  p.free_head_out = data<int32_t>(d, a[11], I, 1, "free_head_out");
  int32_t* flags = data_or_null<int32_t>(d, a[12], I, 1, "flags");
  if (table.dim() != 2 || table.size(0) != B) wrong("table", "[batch, max_pages] is wanted");
  p.max_pages = int32(table.size(1), "table");
  void* s = stream_of(length, a[13]);
  auto f = entry<decltype(&buddy_page_plan)>(a[0]);
  return called(d, [&] { return f(&p, flags, s); });
}

// q, k, pos, cos, sin, q_out, k_out, q_gain, k_gain, eps; with `axes`, pos [axes, tokens]
buddy_qk_rows rows_of(Device& d, PyObject* const* a, buddy_rope_axes* axes = nullptr) {
  const at::Tensor& k = tensor(a[1], "k");
  const ScalarType type = k.scalar_type();
  const auto F = ScalarType::Float;
  if (k.dim() != 3 || dtype_of(type) < 0) wrong("k", "[tokens, heads, head_dim] of fp32 or bf16 is wanted");
  const int64_t T = k.size(0), nkv = k.size(1), hd = k.size(2);
  buddy_qk_rows r{};
  r.n_tok = int32(T, "k");
  r.n_kv_heads = int32(nkv, "k");
  r.head_dim = int32(hd, "k");
  r.dtype = dtype_of(type);
  r.eps = real(a[9]);
  r.k = k.data_ptr();
  r.k_stride = heads(d, k, type, T, nkv, hd, "k");
  if (a[6] != Py_None) {
    const at::Tensor& t = tensor(a[6], "k_out");
    r.k_out_stride = heads(d, t, type, T, nkv, hd, "k_out");
    r.k_out = t.data_ptr();
  }
  if (a[0] != Py_None) {
    const at::Tensor& q = tensor(a[0], "q");
    if (q.dim() != 3) wrong("q", "[tokens, heads, head_dim] is wanted");
    r.n_q_heads = int32(q.size(1), "q");
    r.q_stride = heads(d, q, type, T, r.n_q_heads, hd, "q");
    r.q = q.data_ptr();
    if (a[5] == Py_None) wrong("q_out", "is wanted with q");
    const at::Tensor& t = tensor(a[5], "q_out");
    r.q_out_stride = heads(d, t, type, T, r.n_q_heads, hd, "q_out");
    r.q_out = r.n_q_heads ? t.data_ptr() : nullptr;
  }
  r.rope_cos = table(d, a[3], hd, "cos", &r.max_pos);
  int32_t rows;
  r.rope_sin = table(d, a[4], hd, "sin", &rows);
  if (rows != r.max_pos) wrong("sin", "as many positions as in cos are wanted");
  r.q_gain = data_or_null<float>(d, a[7], F, hd, "q_gain");
  r.k_gain = data_or_null<float>(d, a[8], F, hd, "k_gain");
  if (!axes) {
    r.pos = data<int32_t>(d, a[2], ScalarType::Int, T, "pos");
    return r;
  }
  const at::Tensor& pos = tensor(a[2], "pos");
  if (pos.scalar_type() != ScalarType::Int || !pos.is_cuda() || pos.dim() != 2 || pos.size(0) != axes->n_axes ||
      pos.size(1) != T || (pos.stride(1) != 1 && T > 1)) {
    PyErr_Format(PyExc_ValueError, "pos: CUDA int32 (%d, %lld) with the tokens of an axis one after the other is wanted",
                 (int)axes->n_axes, (long long)T);
    throw Failed{};
  }
  d.take(pos, "pos");
  r.pos = static_cast<const int32_t*>(pos.data_ptr());
  axes->pos_stride = pos.stride(0);
  return r;
}

// What a RopeAxes' address stands for: the axes, and the head dimension that they are of.
struct AxesOf {
  buddy_rope_axes axes;
  int32_t head_dim;
};
buddy_qk_rows rows_with_axes(Device& d, PyObject* const* a, PyObject* address, buddy_rope_axes* axes) {
  const AxesOf* const given = entry<const AxesOf*>(address);
  *axes = given->axes;
  const buddy_qk_rows r = rows_of(d, a, axes);
  if (r.head_dim != given->head_dim) wrong("axes", "axes of the head dimension of k are wanted");
  return r;
}

// entry, the ten of rows_of, flags, stream
PyObject* qk_norm_rope(PyObject* const* a) {
  Device d;
  const buddy_qk_rows r = rows_of(d, a + 1);
  int32_t* flags = data_or_null<int32_t>(d, a[11], ScalarType::Int, 1, "flags");
  void* s = stream_of(tensor(a[2], "k"), a[12]);
  auto f = entry<decltype(&buddy_qk_norm_rope)>(a[0]);
  return called(d, [&] { return f(&r, flags, s); });
}

// entry, the ten of rows_of, flags, stream, axes
PyObject* qk_norm_rope_axes(PyObject* const* a) {
  Device d;
  buddy_rope_axes axes;
  const buddy_qk_rows r = rows_with_axes(d, a + 1, a[13], &axes);
  int32_t* flags = data_or_null<int32_t>(d, a[11], ScalarType::Int, 1, "flags");
  void* s = stream_of(tensor(a[2], "k"), a[12]);
  auto f = entry<decltype(&buddy_qk_norm_rope_axes)>(a[0]);
  return called(d, [&] { return f(&r, &axes, flags, s); });
}

// The cache's address, the ten of rows_of, v, slot, flags, stream
struct Append {
  const buddy_kv4_cache* c;
  buddy_qk_rows r;
  const void* v;
  int64_t v_stride;
  const int64_t* slot;
  int32_t* flags;
  void* stream;
};
Append append_of(Device& d, PyObject* const* a, PyObject* address = nullptr, buddy_rope_axes* axes = nullptr) {
  Append x;
  x.c = &pages(d, a[0])->c;
  x.r = axes ? rows_with_axes(d, a + 1, address, axes) : rows_of(d, a + 1);
  const at::Tensor& k = tensor(a[2], "k");
  const at::Tensor& v = tensor(a[11], "v");
  x.v_stride = heads(d, v, k.scalar_type(), x.r.n_tok, x.r.n_kv_heads, x.r.head_dim, "v");
  x.slot = data<int64_t>(d, a[12], ScalarType::Long, x.r.n_tok, "slot");
  x.flags = data_or_null<int32_t>(d, a[13], ScalarType::Int, 1, "flags");
  x.stream = stream_of(k, a[14]);
  x.v = v.data_ptr();
  return x;
}

// entry, those of append_of
PyObject* kv4_append(PyObject* const* a) {
  Device d;
  const Append x = append_of(d, a + 1);
  auto f = entry<decltype(&buddy_kv4_append)>(a[0]);
  return called(d, [&] { return f(x.c, &x.r, x.v, x.v_stride, x.slot, x.flags, x.stream); });
}

// entry, those of append_of, axes
PyObject* kv4_append_axes(PyObject* const* a) {
  Device d;
  buddy_rope_axes axes;
  const Append x = append_of(d, a + 1, a[16], &axes);
  auto f = entry<decltype(&buddy_kv4_append_axes)>(a[0]);
  return called(d, [&] { return f(x.c, &x.r, &axes, x.v, x.v_stride, x.slot, x.flags, x.stream); });
}

// entry, cache's address, slot, k_out, v_out, flags, stream
PyObject* kv4_read(PyObject* const* a) {
  Device d;
  const buddy_kv4_cache* const c = &pages(d, a[1])->c;
  const at::Tensor& slot = vec(d, a[2], ScalarType::Long, 0, "slot");
  PyObject* const out = a[3] != Py_None ? a[3] : a[4];
  const ScalarType type = out == Py_None ? ScalarType::Undefined : tensor(out, "k_out, v_out").scalar_type();
  const int32_t dtype = dtype_of(type), n = int32(slot.numel(), "slot");
  if (dtype < 0) wrong("k_out, v_out", "fp32, fp16 or bf16 is wanted");
  const int64_t size = (int64_t)n * c->n_kv_heads * c->head_dim;
  void* k = data_or_null<void>(d, a[3], type, size, "k_out");
  void* v = data_or_null<void>(d, a[4], type, size, "v_out");
  int32_t* flags = data_or_null<int32_t>(d, a[5], ScalarType::Int, 1, "flags");
  void* s = stream_of(slot, a[6]);
  const int64_t* at = static_cast<int64_t*>(slot.data_ptr());
  auto f = entry<decltype(&buddy_kv4_read)>(a[0]);
  return called(d, [&] { return f(c, n, at, dtype, k, v, flags, s); });
}

// entry, cache's address, q, kv_len, table, out, row_start, max_new, scale, flags, workspace, stream
PyObject* kv4_attention(PyObject* const* a) {
  Device d;
  const auto I = ScalarType::Int;
  const buddy_kv4_cache* const c = &pages(d, a[1])->c;
  const at::Tensor& q = tensor(a[2], "q");
  const at::Tensor& out = tensor(a[5], "out");
  const at::Tensor& kv_len = tensor(a[3], "kv_len");
  if (q.dim() != 3 || q.size(2) != c->head_dim) wrong("q", "[tokens, heads, head_dim of the cache] is wanted");
  buddy_kv4_attention_args p{};
  const int64_t B = kv_len.numel();
  p.batch = int32(B, "kv_len");
  p.n_tok = int32(q.size(0), "q");
  p.n_q_heads = int32(q.size(1), "q");
  p.max_new = int32(a[7]);
  p.scale = real(a[8]);
  p.q_dtype = dtype_of(q.scalar_type());
  p.out_dtype = dtype_of(out.scalar_type());
  p.q_stride = heads(d, q, q.scalar_type(), p.n_tok, p.n_q_heads, c->head_dim, "q");
  p.out_stride = heads(d, out, out.scalar_type(), p.n_tok, p.n_q_heads, c->head_dim, "out");
  p.q = q.data_ptr();
  p.out = out.data_ptr();
  p.row_start = data_or_null<int32_t>(d, a[6], I, B + 1, "row_start");
  p.kv_len = data<int32_t>(d, a[3], I, B, "kv_len");
  const at::Tensor& table = vec(d, a[4], I, 0, "table");
  if (table.dim() != 2 || table.size(0) != B) wrong("table", "[batch, max_pages] is wanted");
  p.max_pages = int32(table.size(1), "table");
  p.table = static_cast<int32_t*>(table.data_ptr());
  const at::Tensor& ws = vec(d, a[10], ScalarType::Byte, 0, "workspace");
  p.workspace = ws.data_ptr();
  p.workspace_bytes = ws.numel();
  int32_t* flags = data_or_null<int32_t>(d, a[9], I, 1, "flags");
  void* s = stream_of(q, a[11]);
  auto f = entry<decltype(&buddy_kv4_attention)>(a[0]);
  return called(d, [&] { return f(c, &p, flags, s); });
}

// kv_len, table, row_start, max_new of a call with `tokens` rows (-1: as many as row_start says)
buddy_kv4_seqs seqs_of(Device& d, PyObject* const* a, int64_t tokens) {
  const auto I = ScalarType::Int;
  const int64_t B = tensor(a[0], "kv_len").numel();
  buddy_kv4_seqs s{};
  s.batch = int32(B, "kv_len");
  s.kv_len = data<int32_t>(d, a[0], I, B, "kv_len");
  const at::Tensor& table = vec(d, a[1], I, 0, "table");
  if (table.dim() != 2 || table.size(0) != B) wrong("table", "[batch, max_pages] is wanted");
  s.max_pages = int32(table.size(1), "table");
  s.table = static_cast<int32_t*>(table.data_ptr());
  s.row_start = data_or_null<int32_t>(d, a[2], I, B + 1, "row_start");
  s.max_new = int32(a[3]);
  s.n_tok = tokens >= 0 ? int32(tokens, "q") : s.row_start ? INT32_MAX : s.batch;
  return s;
}

// The keys' bounds of a cache: half [n_pages, n_kv_heads, 2, head_dim].
void* bounds_of(Device& d, PyObject* o, const buddy_kv4_cache* c) {
  const at::Tensor& t = vec(d, o, ScalarType::Half, 0, "bounds");
  if (t.dim() != 4 || t.size(0) != c->n_pages || t.size(1) != c->n_kv_heads || t.size(2) != 2 || t.size(3) != c->head_dim)
    wrong("bounds", "[n_pages, n_kv, 2, head_dim] of the cache is wanted");
  return t.data_ptr();
}

// entry, cache's address, bounds, kv_len, table, row_start, max_new, flags, stream
PyObject* kv4_bounds(PyObject* const* a) {
  Device d;
  const buddy_kv4_cache* const c = &pages(d, a[1])->c;
  void* const bounds = bounds_of(d, a[2], c);
  const buddy_kv4_seqs s = seqs_of(d, a + 3, -1);
  int32_t* flags = data_or_null<int32_t>(d, a[7], ScalarType::Int, 1, "flags");
  void* stream = stream_of(tensor(a[2], "bounds"), a[8]);
  auto f = entry<decltype(&buddy_kv4_bounds)>(a[0]);
  return called(d, [&] { return f(c, &s, bounds, flags, stream); });
}

// The lists of pages of a call's tokens, [tokens, n_kv_heads, pages]: entries of one.
int32_t* lists_of(Device& d, PyObject* o, const buddy_kv4_cache* c, int64_t tokens, int32_t* entries) {
  const at::Tensor& t = vec(d, o, ScalarType::Int, 0, "pages");
  if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != c->n_kv_heads) wrong("pages", "[tokens, n_kv, budget] is wanted");
  *entries = int32(t.size(2), "pages");
  return static_cast<int32_t*>(t.data_ptr());
}

// entry, cache's address, q, bounds, kv_len, table, row_start, max_new, pages, visible, first, last, flags, stream
PyObject* kv4_select(PyObject* const* a) {
  Device d;
  const buddy_kv4_cache* const c = &pages(d, a[1])->c;
  const at::Tensor& q = tensor(a[2], "q");
  if (q.dim() != 3 || q.size(2) != c->head_dim) wrong("q", "[tokens, heads, head_dim of the cache] is wanted");
  buddy_kv4_select_args p{};
  p.n_q_heads = int32(q.size(1), "q");
  p.q_dtype = dtype_of(q.scalar_type());
  p.q_stride = heads(d, q, q.scalar_type(), q.size(0), p.n_q_heads, c->head_dim, "q");
  p.q = q.data_ptr();
  p.bounds = bounds_of(d, a[3], c);
  p.s = seqs_of(d, a + 4, q.size(0));
  p.pages = lists_of(d, a[8], c, q.size(0), &p.budget);
  p.visible = data<int32_t>(d, a[9], ScalarType::Int, q.size(0), "visible");
  p.first = int32(a[10]);
  p.last = int32(a[11]);
  int32_t* flags = data_or_null<int32_t>(d, a[12], ScalarType::Int, 1, "flags");
  void* s = stream_of(q, a[13]);
  auto f = entry<decltype(&buddy_kv4_select)>(a[0]);
  return called(d, [&] { return f(c, &p, flags, s); });
}

// entry, cache's address, q, visible, pages, out, scale, flags, workspace, stream
PyObject* kv4_attention_pages(PyObject* const* a) {
  Device d;
  const auto I = ScalarType::Int;
  const buddy_kv4_cache* const c = &pages(d, a[1])->c;
  const at::Tensor& q = tensor(a[2], "q");
  const at::Tensor& out = tensor(a[5], "out");
  if (q.dim() != 3 || q.size(2) != c->head_dim) wrong("q", "[tokens, heads, head_dim of the cache] is wanted");
  buddy_kv4_attention_args p{};
  p.batch = p.n_tok = int32(q.size(0), "q");
  p.n_q_heads = int32(q.size(1), "q");
  p.max_new = 1;
  p.scale = real(a[6]);
  p.q_dtype = dtype_of(q.scalar_type());
  p.out_dtype = dtype_of(out.scalar_type());
  p.q_stride = heads(d, q, q.scalar_type(), p.n_tok, p.n_q_heads, c->head_dim, "q");
  p.out_stride = heads(d, out, out.scalar_type(), p.n_tok, p.n_q_heads, c->head_dim, "out");
  p.q = q.data_ptr();
  p.out = out.data_ptr();
  p.kv_len = data<int32_t>(d, a[3], I, p.n_tok, "visible");
  p.table = lists_of(d, a[4], c, p.n_tok, &p.max_pages);
  const at::Tensor& ws = vec(d, a[8], ScalarType::Byte, 0, "workspace");
  p.workspace = ws.data_ptr();
  p.workspace_bytes = ws.numel();
  int32_t* flags = data_or_null<int32_t>(d, a[7], I, 1, "flags");
  void* s = stream_of(q, a[9]);
  auto f = entry<decltype(&buddy_kv4_attention_pages)>(a[0]);
  return called(d, [&] { return f(c, &p, flags, s); });
}

template <int N, PyObject* (*F)(PyObject* const*)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<N, F>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<14, page_plan>("page_plan"),         method<13, qk_norm_rope>("qk_norm_rope"),
                         method<16, kv4_append>("kv4_append"),       method<7, kv4_read>("kv4_read"),
                         method<12, kv4_attention>("kv4_attention"), method<2, stream_for_workspace>("stream_for_workspace"),
                         method<14, qk_norm_rope_axes>("qk_norm_rope_axes"),
                         method<17, kv4_append_axes>("kv4_append_axes"),
                         method<9, kv4_bounds>("kv4_bounds"),
                         method<14, kv4_select>("kv4_select"),
                         method<10, kv4_attention_pages>("kv4_attention_pages"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
