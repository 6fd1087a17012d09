// The way from torch tensors to the calls of the 8-bit attention path (include/ptq.h): checks, pointers, strides and the current
// stream, nothing else.  These calls are made for every layer and token, where 6 to 10 us of an interpreted binding were more than
// the kernels take; here it is about one.  binding.py has their Python signatures; every function returns the call's status.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ptq.h"

namespace {

struct Refused {};   // the Python error is set

[[noreturn]] void refuse(PyObject* type, const char* why) {
  PyErr_SetString(type, why);
  throw Refused{};
}
#define PTQ_CHECK(cond) \
  do {                  \
    if (!(cond)) refuse(PyExc_AssertionError, #cond); \
  } while (0)

using Tensor = at::Tensor;

const Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "a tensor is expected");
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse(PyExc_ValueError, "libptq takes device tensors only");
  return t;
}
// nullptr for None
const Tensor* optional(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
void* ptr(const Tensor& t) { return t.data_ptr(); }
void* ptr(const Tensor* t) { return t ? t->data_ptr() : nullptr; }
template <class T>
T* as(const Tensor& t) { return static_cast<T*>(t.data_ptr()); }

int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused{};
  return v != 0;
}

// The current stream, of the current device: all tensors have to be there.  (Asking for it twice would take 0.4 us.)
const Tensor* address_of(const Tensor& t) { return &t; }
const Tensor* address_of(const Tensor* t) { return t; }
template <class... T>
ptq_stream stream_of(const T&... t) {
  const auto current = c10::hip::getCurrentHIPStream();
  for (const Tensor* p : {address_of(t)...})
    if (p && p->device().index() != current.device_index()) refuse(PyExc_ValueError, "tensors of another device than the current one");
  return current.stream();
}

// storage types that the library does not know become its own status
bool dtype_of(const Tensor& t, ptq_dtype& d) {
  switch (t.scalar_type()) {
    case at::kFloat: d = PTQ_F32; return true;
    case at::kBFloat16: d = PTQ_BF16; return true;
    case at::kDouble: d = PTQ_F64; return true;
    default: return false;
  }
}

// the caller's workspace, or a new one of the size the call needs
struct Workspace {
  Tensor own;
  void* at = nullptr;
  size_t bytes = 0;
  Workspace(const Tensor* given, const Tensor& like, ptq_op op, int64_t m, int64_t n, int64_t t, int64_t block) {
    if (!given) {
      if (ptq_workspace_bytes(op, m, n, t, block, &bytes) != PTQ_OK || bytes == 0) return;
      own = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
      at = own.data_ptr();
    } else {
      at = given->data_ptr();
      bytes = given->nbytes();
    }
  }
};

template <class F>
PyObject* status_of(F&& call) {
  try {
    return PyLong_FromLong(call());
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
// the library's call, without the interpreter's lock
template <class F>
ptq_status released(F&& call) {
  ptq_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return rc;
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return n == want;
}

// X, codes, scales, gamma, residual, residual_out, eps, normalize
PyObject* rmsnorm_quantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 8)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &X = tensor(a[0]), &codes = tensor(a[1]), &scales = tensor(a[2]);
    const Tensor *gamma = optional(a[3]), *residual = optional(a[4]), *out = optional(a[5]);
    const double eps = number(a[6]);
    const int normalize = truth(a[7]);
    const ptq_stream s = stream_of(X, codes, scales, gamma, residual, out);
    PTQ_CHECK(X.dim() == 2 && X.stride(1) == 1);
    const int64_t t = X.size(0), n = X.size(1);
    PTQ_CHECK(codes.scalar_type() == at::kChar && codes.dim() == 2 && codes.size(0) == t && codes.size(1) == n && codes.stride(1) == 1);
    PTQ_CHECK(scales.scalar_type() == at::kFloat && scales.is_contiguous() && scales.numel() == t);
    PTQ_CHECK(!gamma || (gamma->scalar_type() == X.scalar_type() && gamma->is_contiguous() && gamma->dim() == 1 && gamma->size(0) == n));
    for (const Tensor* r : {residual, out})
      PTQ_CHECK(!r || (r->scalar_type() == X.scalar_type() && r->dim() == 2 && r->size(0) == t && r->size(1) == n && r->stride(1) == 1));
    ptq_dtype dt;
    if (!dtype_of(X, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_rmsnorm_quantize(ptr(X), dt, X.stride(0), t, n, ptr(residual), residual ? residual->stride(0) : 0, ptr(out),
                                  out ? out->stride(0) : 0, ptr(gamma), eps, normalize, as<int8_t>(codes), codes.stride(0),
                                  as<float>(scales), s);
    });
  });
}

// A, a_scales, W, w_scales, O, bias, ws
PyObject* int8_linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 7)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &A = tensor(a[0]), &as_ = tensor(a[1]), &W = tensor(a[2]), &ws_ = tensor(a[3]), &O = tensor(a[4]);
    const Tensor *bias = optional(a[5]), *ws = optional(a[6]);
    const ptq_stream s = stream_of(A, as_, W, ws_, O, bias, ws);
    PTQ_CHECK(A.scalar_type() == at::kChar && A.dim() == 2 && A.stride(1) == 1);
    PTQ_CHECK(W.scalar_type() == at::kChar && W.dim() == 2 && W.stride(1) == 1 && W.size(1) == A.size(1));
    const int64_t t = A.size(0), n = A.size(1), m = W.size(0);
    PTQ_CHECK(as_.scalar_type() == at::kFloat && as_.is_contiguous() && as_.numel() == t);
    PTQ_CHECK(ws_.scalar_type() == at::kFloat && ws_.is_contiguous() && ws_.numel() == m);
    PTQ_CHECK(!bias || (bias->scalar_type() == at::kFloat && bias->is_contiguous() && bias->numel() == m));
    PTQ_CHECK(O.dim() == 2 && O.size(0) == t && O.size(1) == m && O.stride(1) == 1);
    PTQ_CHECK(!ws || ws->is_contiguous());
    ptq_dtype dt;
    if (!dtype_of(O, dt)) return PTQ_ERR_DTYPE;
    const Workspace w(ws, A, PTQ_OP_INT8_LINEAR, m, n, t, 0);
    return released([&] {
      return ptq_int8_linear(as<int8_t>(A), A.stride(0), as<float>(as_), t, as<int8_t>(W), W.stride(0), as<float>(ws_), m, n,
                             static_cast<const float*>(ptr(bias)), ptr(O), dt, O.stride(0), w.at, w.bytes, s);
    });
  });
}

struct Cache { int64_t pages, heads, page; };
Cache cache_of(const Tensor& codes, const Tensor& scales, const Tensor& zeros, int64_t bits, int64_t d) {
  PTQ_CHECK(codes.scalar_type() == at::kByte && codes.is_contiguous() && codes.dim() == 5 && codes.size(0) == 2);
  const Cache c{codes.size(1), codes.size(2), codes.size(3)};
  PTQ_CHECK(codes.size(4) == d * bits / 8);
  auto grid = [&](const Tensor& g) {
    return g.is_contiguous() && g.dim() == 4 && g.size(0) == 2 && g.size(1) == c.pages && g.size(2) == c.heads && g.size(3) == c.page;
  };
  PTQ_CHECK(scales.scalar_type() == at::kFloat && grid(scales));
  PTQ_CHECK(zeros.scalar_type() == at::kByte && grid(zeros));
  return c;
}
bool whole_numbers(const Tensor& t, int64_t n) { return t.scalar_type() == at::kInt && t.is_contiguous() && t.numel() == n; }
bool table_ok(const Tensor& t) { return t.scalar_type() == at::kInt && t.is_contiguous() && t.dim() == 2; }

// K, V, slots, bits, codes, scales, zeros
PyObject* kv_cache_write(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 7)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &K = tensor(a[0]), &V = tensor(a[1]), &slots = tensor(a[2]), &codes = tensor(a[4]), &scales = tensor(a[5]), &zeros = tensor(a[6]);
    const int64_t bits = whole(a[3]);
    const ptq_stream s = stream_of(K, V, slots, codes, scales, zeros);
    PTQ_CHECK(K.dim() == 3 && K.stride(2) == 1 && V.stride(2) == 1 && V.sizes() == K.sizes() && V.scalar_type() == K.scalar_type());
    const int64_t t = K.size(0), heads = K.size(1), d = K.size(2);
    const Cache c = cache_of(codes, scales, zeros, bits, d);
    PTQ_CHECK(c.heads == heads);
    PTQ_CHECK(whole_numbers(slots, t));
    ptq_dtype dt;
    if (!dtype_of(K, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_kv_cache_write(ptr(K), K.stride(0), K.stride(1), ptr(V), V.stride(0), V.stride(1), dt, t, heads, d, as<int32_t>(slots), (int)bits,
                                as<uint8_t>(codes), as<float>(scales), as<uint8_t>(zeros), c.pages, c.page, s);
    });
  });
}

// codes, scales, zeros, bits, table, cu_kv, max_kv, K, V
PyObject* kv_cache_read(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 9)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &codes = tensor(a[0]), &scales = tensor(a[1]), &zeros = tensor(a[2]), &table = tensor(a[4]), &cu = tensor(a[5]),
                 &K = tensor(a[7]), &V = tensor(a[8]);
    const int64_t bits = whole(a[3]), max_kv = whole(a[6]);
    const ptq_stream s = stream_of(codes, scales, zeros, table, cu, K, V);
    PTQ_CHECK(K.dim() == 3 && K.stride(2) == 1 && V.stride(2) == 1 && V.sizes() == K.sizes() && V.scalar_type() == K.scalar_type());
    const int64_t rows = K.size(0), heads = K.size(1), d = K.size(2);
    const Cache c = cache_of(codes, scales, zeros, bits, d);
    PTQ_CHECK(c.heads == heads);
    PTQ_CHECK(table_ok(table));
    const int64_t b = table.size(0);
    PTQ_CHECK(whole_numbers(cu, b + 1));
    ptq_dtype dt;
    if (!dtype_of(K, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_kv_cache_read(as<uint8_t>(codes), as<float>(scales), as<uint8_t>(zeros), c.pages, c.page, heads, d, (int)bits, as<int32_t>(table),
                               table.size(1), b, as<int32_t>(cu), rows, max_kv, ptr(K), K.stride(0), K.stride(1), ptr(V), V.stride(0),
                               V.stride(1), dt, s);
    });
  });
}

// Q, cu_q, max_q, codes, scales, zeros, bits, table, kv_lens, max_kv, softmax_scale, O, causal, window, ws
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 15)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &Q = tensor(a[0]), &cu = tensor(a[1]), &codes = tensor(a[3]), &scales = tensor(a[4]), &zeros = tensor(a[5]), &table = tensor(a[7]),
                 &lens = tensor(a[8]), &O = tensor(a[11]);
    const Tensor* ws = optional(a[14]);
    const int64_t max_q = whole(a[2]), bits = whole(a[6]), max_kv = whole(a[9]), window = whole(a[13]);
    const double scale = number(a[10]);
    const int causal = truth(a[12]);
    const ptq_stream s = stream_of(Q, cu, codes, scales, zeros, table, lens, O, ws);
    PTQ_CHECK(Q.dim() == 3 && Q.stride(2) == 1 && O.stride(2) == 1 && O.sizes() == Q.sizes() && O.scalar_type() == Q.scalar_type());
    const int64_t t = Q.size(0), hq = Q.size(1), d = Q.size(2);
    const Cache c = cache_of(codes, scales, zeros, bits, d);
    PTQ_CHECK(table_ok(table));
    const int64_t b = table.size(0);
    PTQ_CHECK(whole_numbers(cu, b + 1));
    PTQ_CHECK(whole_numbers(lens, b));
    PTQ_CHECK(!ws || ws->is_contiguous());
    ptq_dtype dt;
    if (!dtype_of(Q, dt)) return PTQ_ERR_DTYPE;
    const Workspace w(ws, Q, PTQ_OP_PAGED_ATTENTION, hq, d, t, max_kv);
    return released([&] {
      return ptq_paged_attention(ptr(Q), dt, Q.stride(0), Q.stride(1), t, hq, d, as<int32_t>(cu), b, max_q, as<uint8_t>(codes), as<float>(scales),
                                 as<uint8_t>(zeros), c.pages, c.page, c.heads, (int)bits, as<int32_t>(table), table.size(1), as<int32_t>(lens),
                                 max_kv, scale, causal, window, ptr(O), O.stride(0), O.stride(1), w.at, w.bytes, s);
    });
  });
}

// X and Y of a rotation, positions and frequencies
void rotary_ok(const Tensor& X, const Tensor& Y, const Tensor& positions, const Tensor& freq) {
  PTQ_CHECK(X.dim() == 3 && X.stride(2) == 1 && Y.sizes() == X.sizes() && Y.stride(2) == 1 && Y.scalar_type() == X.scalar_type());
  PTQ_CHECK(whole_numbers(positions, X.size(0)));
  PTQ_CHECK(freq.scalar_type() == at::kDouble && freq.is_contiguous() && freq.dim() == 1);
}

// X, positions, freq, Y, scale, interleaved
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 6)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &X = tensor(a[0]), &positions = tensor(a[1]), &freq = tensor(a[2]), &Y = tensor(a[3]);
    const double scale = number(a[4]);
    const int interleaved = truth(a[5]);
    const ptq_stream s = stream_of(X, positions, freq, Y);
    rotary_ok(X, Y, positions, freq);
    ptq_dtype dt;
    if (!dtype_of(X, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_rotary(ptr(X), X.stride(0), X.stride(1), dt, X.size(0), X.size(1), X.size(2), as<int32_t>(positions), as<double>(freq), 2 * freq.numel(),
                        scale, interleaved, ptr(Y), Y.stride(0), Y.stride(1), s);
    });
  });
}

// Q, K, V, positions, freq, slots, bits, codes, scales, zeros, Q_out, scale, interleaved
PyObject* rotary_kv_cache_write(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 13)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &Q = tensor(a[0]), &K = tensor(a[1]), &V = tensor(a[2]), &positions = tensor(a[3]), &freq = tensor(a[4]), &slots = tensor(a[5]),
                 &codes = tensor(a[7]), &scales = tensor(a[8]), &zeros = tensor(a[9]), &O = tensor(a[10]);
    const int64_t bits = whole(a[6]);
    const double scale = number(a[11]);
    const int interleaved = truth(a[12]);
    const ptq_stream s = stream_of(Q, K, V, positions, freq, slots, codes, scales, zeros, O);
    rotary_ok(Q, O, positions, freq);
    PTQ_CHECK(K.dim() == 3 && K.stride(2) == 1 && V.sizes() == K.sizes() && V.stride(2) == 1 && K.scalar_type() == Q.scalar_type() && V.scalar_type() == Q.scalar_type());
    const int64_t t = K.size(0), heads = K.size(1), d = K.size(2);
    PTQ_CHECK(Q.size(0) == t && Q.size(2) == d);
    const Cache c = cache_of(codes, scales, zeros, bits, d);
    PTQ_CHECK(c.heads == heads);
    PTQ_CHECK(whole_numbers(slots, t));
    ptq_dtype dt;
    if (!dtype_of(Q, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_rotary_kv_cache_write(ptr(Q), Q.stride(0), Q.stride(1), Q.size(1), ptr(K), K.stride(0), K.stride(1), ptr(V), V.stride(0), V.stride(1), dt,
                                       t, heads, d, as<int32_t>(positions), as<double>(freq), 2 * freq.numel(), scale, interleaved, as<int32_t>(slots),
                                       (int)bits, as<uint8_t>(codes), as<float>(scales), as<uint8_t>(zeros), c.pages, c.page, ptr(O), O.stride(0),
                                       O.stride(1), s);
    });
  });
}

// from_codes, from_scales, from_zeros, source, codes, scales, zeros, target
PyObject* kv_cache_copy_pages(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 8)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &fc = tensor(a[0]), &fs = tensor(a[1]), &fz = tensor(a[2]), &source = tensor(a[3]), &codes = tensor(a[4]), &scales = tensor(a[5]),
                 &zeros = tensor(a[6]), &target = tensor(a[7]);
    const ptq_stream s = stream_of(fc, fs, fz, source, codes, scales, zeros, target);
    PTQ_CHECK(fc.dim() == 5 && codes.dim() == 5 && fc.size(4) == codes.size(4));
    const Cache from = cache_of(fc, fs, fz, 8, fc.size(4)), to = cache_of(codes, scales, zeros, 8, codes.size(4));
    PTQ_CHECK(from.heads == to.heads && from.page == to.page);
    const int64_t n = source.numel();
    PTQ_CHECK(whole_numbers(source, n) && whole_numbers(target, n));
    return released([&] {
      return ptq_kv_cache_copy_pages(as<uint8_t>(fc), as<float>(fs), as<uint8_t>(fz), from.pages, as<uint8_t>(codes), as<float>(scales), as<uint8_t>(zeros),
                                     to.pages, to.page, to.heads, codes.size(4), as<int32_t>(source), as<int32_t>(target), n, s);
    });
  });
}

// Q, K, V, cu, max_n, softmax_scale, O, causal, window
PyObject* prompt_attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 9)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &Q = tensor(a[0]), &K = tensor(a[1]), &V = tensor(a[2]), &cu = tensor(a[3]), &O = tensor(a[6]);
    const int64_t max_n = whole(a[4]), window = whole(a[8]);
    const double scale = number(a[5]);
    const int causal = truth(a[7]);
    const ptq_stream s = stream_of(Q, K, V, cu, O);
    PTQ_CHECK(Q.dim() == 3 && Q.stride(2) == 1 && O.stride(2) == 1 && O.sizes() == Q.sizes() && O.scalar_type() == Q.scalar_type());
    PTQ_CHECK(K.dim() == 3 && K.stride(2) == 1 && V.stride(2) == 1 && V.sizes() == K.sizes() && K.scalar_type() == Q.scalar_type() &&
              V.scalar_type() == Q.scalar_type());
    PTQ_CHECK(K.size(0) == Q.size(0) && K.size(2) == Q.size(2));
    PTQ_CHECK(cu.scalar_type() == at::kInt && cu.is_contiguous() && cu.numel() >= 1);
    ptq_dtype dt;
    if (!dtype_of(Q, dt)) return PTQ_ERR_DTYPE;
    return released([&] {
      return ptq_prompt_attention(ptr(Q), Q.stride(0), Q.stride(1), ptr(K), K.stride(0), K.stride(1), ptr(V), V.stride(0), V.stride(1), dt, Q.size(0),
                                  Q.size(1), K.size(1), Q.size(2), as<int32_t>(cu), cu.numel() - 1, max_n, scale, causal, window, ptr(O), O.stride(0),
                                  O.stride(1), s);
    });
  });
}

// Q, cu_q, max_q, codes, scales, zeros, bits, table, kv_lens, max_kv, cu_groups, shared, max_shared, softmax_scale, O, causal, ws
PyObject* paged_attention_shared(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (!count_is(count, 17)) return nullptr;
  return status_of([&]() -> ptq_status {
    const Tensor &Q = tensor(a[0]), &cu = tensor(a[1]), &codes = tensor(a[3]), &scales = tensor(a[4]), &zeros = tensor(a[5]), &table = tensor(a[7]),
                 &lens = tensor(a[8]), &cu_groups = tensor(a[10]), &shared = tensor(a[11]), &O = tensor(a[14]);
    const Tensor* ws = optional(a[16]);
    const int64_t max_q = whole(a[2]), bits = whole(a[6]), max_kv = whole(a[9]), max_shared = whole(a[12]);
    const double scale = number(a[13]);
    const int causal = truth(a[15]);
    const ptq_stream s = stream_of(Q, cu, codes, scales, zeros, table, lens, cu_groups, shared, O, ws);
    PTQ_CHECK(Q.dim() == 3 && Q.stride(2) == 1 && O.stride(2) == 1 && O.sizes() == Q.sizes() && O.scalar_type() == Q.scalar_type());
    const int64_t t = Q.size(0), hq = Q.size(1), d = Q.size(2);
    const Cache c = cache_of(codes, scales, zeros, bits, d);
    PTQ_CHECK(table_ok(table));
    const int64_t b = table.size(0), groups = shared.numel();
    PTQ_CHECK(whole_numbers(cu, b + 1));
    PTQ_CHECK(whole_numbers(lens, b));
    PTQ_CHECK(whole_numbers(cu_groups, groups + 1) && whole_numbers(shared, groups));
    PTQ_CHECK(!ws || ws->is_contiguous());
    ptq_dtype dt;
    if (!dtype_of(Q, dt)) return PTQ_ERR_DTYPE;
    const Workspace w(ws, Q, PTQ_OP_SHARED_ATTENTION, hq, d, t, max_kv);
    return released([&] {
      return ptq_paged_attention_shared(ptr(Q), dt, Q.stride(0), Q.stride(1), t, hq, d, as<int32_t>(cu), b, max_q, as<uint8_t>(codes), as<float>(scales),
                                        as<uint8_t>(zeros), c.pages, c.page, c.heads, (int)bits, as<int32_t>(table), table.size(1), as<int32_t>(lens),
                                        max_kv, as<int32_t>(cu_groups), as<int32_t>(shared), groups, max_shared, scale, causal, ptr(O), O.stride(0),
                                        O.stride(1), w.at, w.bytes, s);
    });
  });
}

#define PTQ_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PTQ_METHOD(rmsnorm_quantize), PTQ_METHOD(int8_linear), PTQ_METHOD(kv_cache_write), PTQ_METHOD(kv_cache_read),
                         PTQ_METHOD(paged_attention), PTQ_METHOD(rotary), PTQ_METHOD(rotary_kv_cache_write), PTQ_METHOD(kv_cache_copy_pages), PTQ_METHOD(prompt_attention), PTQ_METHOD(paged_attention_shared), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tokens", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tokens(void) { return PyModule_Create(&module); }
