// Native part of the Python binding (api.py) for the calls that are shorter on the device than their submission from Python:
// the checks, the result tensors, the addresses and the call into the library in one step.  The library sees addresses only,
// so every tensor is held against what the kernels will read or write of it.  Everything that is not the usual case (other
// argument types, tensors that do not fit, another device than the current one) goes back to Python, which says what is wrong
// or makes the call itself.  The library's functions are handed over as addresses by api.py, so that they come from the
// library it has loaded (bind).
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "covspec.h"

namespace {

using CorrectFn = int (*)(int, int, int, long long, const void*, const void*, const int*, const float*, float, float*, int*,
                          float*, float*, int*, void*);
using CandidatesFn = int (*)(int, int, int, long long, const void*, const int*, const int*, int, int*, void*);
using StaticFn = int (*)(int, int, int, const void*, const int*, const void*, const int*, float*, void*);
CorrectFn g_correct = nullptr;
CandidatesFn g_candidates = nullptr;
StaticFn g_static = nullptr;
decltype(&covspec_cache_write) g_write = nullptr;
decltype(&covspec_cache_read) g_read = nullptr;
decltype(&covspec_cache_attend) g_attend = nullptr;
decltype(&covspec_edit_logits) g_edit = nullptr;

PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long f[7] = {};
  if (!PyArg_ParseTuple(args, "KKKKKKK", f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6)) return nullptr;
  auto put = [](auto& to, unsigned long long from) {
    to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(static_cast<uintptr_t>(from));
  };
  put(g_correct, f[0]);
  put(g_candidates, f[1]);
  put(g_static, f[2]);
  put(g_write, f[3]);
  put(g_read, f[4]);
  put(g_attend, f[5]);
  put(g_edit, f[6]);
  Py_RETURN_NONE;
}

// COVSPEC_F32, COVSPEC_BF16, COVSPEC_F16 (covspec.h); -1: no logit type
int dtype_code(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return 0;
    case at::kBFloat16: return 1;
    case at::kHalf: return 2;
    default: return -1;
  }
}
// Dense memory of at least `least` elements of this type on the call's device.
bool fits(const at::Tensor& t, at::ScalarType type, const at::Device& dev, long long least) {
  return t.device() == dev && t.scalar_type() == type && t.is_contiguous() && t.numel() >= least;
}
// The call's tensors lie on the current device, whose stream takes the launch.
bool on_current_device(const at::Tensor& t) { return t.is_cuda() && t.device().index() == c10::cuda::current_device(); }
bool is_int(long long v) { return v >= INT_MIN && v <= INT_MAX; }
bool int_arg(PyObject* o, long long& v) {
  v = PyLong_AsLongLong(o);
  return !(v == -1 && PyErr_Occurred());
}
// The memory of a C-contiguous int32 array; released when the view goes.
struct IntArray {
  Py_buffer view{};
  bool held = false;
  bool get(PyObject* o, bool writable) {
    if (PyObject_GetBuffer(o, &view, PyBUF_C_CONTIGUOUS | (writable ? PyBUF_WRITABLE : 0))) return false;
    held = true;
    if (view.itemsize != 4) { PyErr_SetString(PyExc_TypeError, "int32 array required"); return false; }
    return true;
  }
  int* data() const { return static_cast<int*>(view.buf); }
  long long size() const { return view.len / 4; }
  ~IntArray() { if (held) PyBuffer_Release(&view); }
};
// The library's call with the interpreter lock released, as ctypes does: a launch may wait for the device's queue.
template <typename F, typename... A>
int call(F f, A... args) {
  int st = 0;
  Py_BEGIN_ALLOW_THREADS
  st = f(args...);
  Py_END_ALLOW_THREADS
  return st;
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// correct(z_draft, z_target, uniforms or None, gamma, drafted or None, vocab) -> (margin, gate, accept, mass, token), or the
// library's status; None where an argument is not of the usual kind.
PyObject* correct(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1]) || !(a[2] == Py_None || THPVariable_Check(a[2])) ||
      !(a[4] == Py_None || THPVariable_Check(a[4])))
    Py_RETURN_NONE;
  const at::Tensor &zd = THPVariable_Unpack(a[0]), &zt = THPVariable_Unpack(a[1]);
  if (!on_current_device(zd) || zd.dim() != 2 || !zd.is_contiguous() || dtype_code(zd) < 0 || !zd.sizes().equals(zt.sizes()) ||
      !fits(zt, zd.scalar_type(), zd.device(), zd.numel()))
    Py_RETURN_NONE;
  const long long rows = zd.size(0), ld = zd.size(1);
  if ((a[2] != Py_None && !fits(THPVariable_Unpack(a[2]), at::kFloat, zd.device(), rows)) ||
      (a[4] != Py_None && !fits(THPVariable_Unpack(a[4]), at::kInt, zd.device(), rows)))
    Py_RETURN_NONE;
  const double gamma = PyFloat_AsDouble(a[3]);
  if (gamma == -1.0 && PyErr_Occurred()) return nullptr;
  long long vocab = ld;
  if (a[5] != Py_None && !int_arg(a[5], vocab)) return nullptr;
  if (!is_int(vocab) || !is_int(rows)) Py_RETURN_NONE;
  const auto f32 = zd.options().dtype(at::kFloat), i32 = zd.options().dtype(at::kInt);
  at::Tensor margin = at::empty({rows}, f32), gate = at::empty({rows}, i32), accept = at::empty({rows}, f32),
             mass = at::empty({rows}, f32), token = at::empty({rows}, i32);
  const void* drafted = a[4] == Py_None ? nullptr : THPVariable_Unpack(a[4]).data_ptr();
  const void* uniforms = a[2] == Py_None ? nullptr : THPVariable_Unpack(a[2]).data_ptr();
  const int st = call(g_correct, dtype_code(zd), (int)rows, (int)vocab, ld, zd.data_ptr(), zt.data_ptr(), static_cast<const int*>(drafted),
                           static_cast<const float*>(uniforms), (float)gamma, static_cast<float*>(margin.data_ptr()),
                           static_cast<int*>(gate.data_ptr()), static_cast<float*>(accept.data_ptr()),
                           static_cast<float*>(mass.data_ptr()), static_cast<int*>(token.data_ptr()), current_stream());
  if (st) return PyLong_FromLong(st);
  PyObject* out = PyTuple_New(5);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(margin)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(gate)));
  PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(std::move(accept)));
  PyTuple_SET_ITEM(out, 3, THPVariable_Wrap(std::move(mass)));
  PyTuple_SET_ITEM(out, 4, THPVariable_Wrap(std::move(token)));
  return out;
  END_HANDLE_TH_ERRORS
}

// candidates(z_draft, fanouts: list of int, off: int32 array of rows + 1, filled in, drafted or None, vocab) -> cand, or the
// library's status; None where an argument is not of the usual kind.
PyObject* candidates(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || !THPVariable_Check(a[0]) || !PyList_CheckExact(a[1]) || !(a[3] == Py_None || THPVariable_Check(a[3]))) Py_RETURN_NONE;
  const at::Tensor& z = THPVariable_Unpack(a[0]);
  if (!on_current_device(z) || z.dim() != 2 || !z.is_contiguous() || dtype_code(z) < 0) Py_RETURN_NONE;
  const long long rows = z.size(0), ld = z.size(1);
  if (a[3] != Py_None && !fits(THPVariable_Unpack(a[3]), at::kInt, z.device(), rows)) Py_RETURN_NONE;
  IntArray off;
  if (!off.get(a[2], true)) return nullptr;
  if (PyList_GET_SIZE(a[1]) != rows || off.size() != rows + 1 || rows < 1) Py_RETURN_NONE;
  long long vocab = ld, total = 0, most = 0;
  if (a[4] != Py_None && !int_arg(a[4], vocab)) return nullptr;
  if (!is_int(vocab) || !is_int(rows)) Py_RETURN_NONE;
  off.data()[0] = 0;
  for (long long r = 0; r < rows; ++r) {
    PyObject* item = PyList_GET_ITEM(a[1], r);
    if (!PyLong_CheckExact(item)) Py_RETURN_NONE;
    int overflow = 0;
    const long long f = PyLong_AsLongLongAndOverflow(item, &overflow);
    if (overflow || f < 0 || f > 0x7fffffff) Py_RETURN_NONE;
    total += f;
    if (total > 0x7fffffff) Py_RETURN_NONE;
    most = r == 0 || f > most ? f : most;
    off.data()[r + 1] = (int)total;
  }
  at::Tensor cand = at::empty({total > 0 ? total : 1}, z.options().dtype(at::kInt));
  const void* drafted = a[3] == Py_None ? nullptr : THPVariable_Unpack(a[3]).data_ptr();
  const int st = call(g_candidates, dtype_code(z), (int)rows, (int)vocab, ld, z.data_ptr(), static_cast<const int*>(drafted),
                              off.data(), (int)most, static_cast<int*>(cand.data_ptr()), current_stream());
  if (st) return PyLong_FromLong(st);
  return THPVariable_Wrap(total ? std::move(cand) : cand.slice(0, 0, 0));
  END_HANDLE_TH_ERRORS
}

// static_score(X, Q, vis, txt: int32 arrays, out) -> the library's status; None where an argument is not of the usual kind.
PyObject* static_score(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1]) || !THPVariable_Check(a[4])) Py_RETURN_NONE;
  IntArray vis, txt;
  if (!vis.get(a[2], false) || !txt.get(a[3], false)) return nullptr;
  const at::Tensor &x = THPVariable_Unpack(a[0]), &q = THPVariable_Unpack(a[1]), &out = THPVariable_Unpack(a[4]);
  const at::ScalarType type = x.scalar_type();
  if (!on_current_device(x) || (type != at::kBFloat16 && type != at::kFloat) || x.dim() != 2 || q.dim() != 2 || x.size(1) != q.size(1) ||
      !is_int(x.size(1)) || vis.size() < 2 || vis.size() != txt.size() || !is_int(vis.size()))
    Py_RETURN_NONE;
  // the library refuses offsets that do not ascend from 0, so the last ones say what is read
  const long long d = x.size(1), rows_x = vis.data()[vis.size() - 1], rows_q = txt.data()[txt.size() - 1];
  if (!fits(x, type, x.device(), rows_x * d) || !fits(q, type, x.device(), rows_q * d) || !fits(out, at::kFloat, x.device(), rows_x))
    Py_RETURN_NONE;
  const int st = call(g_static, type == at::kBFloat16 ? 1 : 0, (int)d, (int)vis.size() - 1, x.data_ptr(), vis.data(), q.data_ptr(),
                      txt.data(), static_cast<float*>(out.data_ptr()), current_stream());
  return PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// ---- the paged cache ----
// A cache's struct, as the address that the PagedCache keeps, and its keys.
bool cache_of(PyObject* address, PyObject* keys, const covspec_cache*& c, const at::Tensor*& k) {
  if (!PyLong_Check(address) || !THPVariable_Check(keys)) return false;
  c = reinterpret_cast<const covspec_cache*>(PyLong_AsVoidPtr(address));
  k = &THPVariable_Unpack(keys);
  return c != nullptr && on_current_device(*k);
}
bool tokens_of(PyObject* const* a, const at::Device& dev, covspec_tokens& t) {
  for (int i = 0; i < 3; ++i)
    if (!THPVariable_Check(a[i])) return false;
  const at::Tensor &offsets = THPVariable_Unpack(a[0]), &lengths = THPVariable_Unpack(a[1]), &table = THPVariable_Unpack(a[2]);
  if (offsets.dim() != 1 || lengths.dim() != 1 || table.dim() != 2) return false;
  const long long batch = lengths.size(0);
  if (!is_int(batch) || !is_int(table.size(1)) || !fits(lengths, at::kInt, dev, batch) || !fits(offsets, at::kInt, dev, batch + 1) ||
      !fits(table, at::kInt, dev, batch * table.size(1)) || table.size(0) < batch)
    return false;
  t = covspec_tokens{(int)batch, static_cast<const int*>(offsets.data_ptr()), static_cast<const int*>(lengths.data_ptr()),
                     static_cast<const int*>(table.data_ptr()), (int)table.size(1), table.size(1)};
  return true;
}
// Rows [n, heads, dim], dense but for the step from row to row.
bool rows_of(const at::Tensor& t, const at::Device& dev, long long heads, long long dim, long long& step) {
  if (t.device() != dev || t.dim() != 3 || t.size(1) != heads || t.size(2) != dim || t.stride(2) != 1 || (heads > 1 && t.stride(1) != dim) ||
      t.size(0) < 1 || !is_int(t.size(0)))
    return false;
  step = t.size(0) > 1 ? t.stride(0) : heads * dim;
  return true;
}

// cache_write(cache, keys, k, v, offsets, lengths, table, rows or None, row_offsets or None) -> the library's status; None where
// an argument is not of the usual kind.
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const covspec_cache* c;
  const at::Tensor* keys;
  covspec_tokens t;
  if (n != 9 || !cache_of(a[0], a[1], c, keys) || !THPVariable_Check(a[2]) || !THPVariable_Check(a[3]) || !tokens_of(a + 4, keys->device(), t)) Py_RETURN_NONE;
  const at::Tensor &k = THPVariable_Unpack(a[2]), &v = THPVariable_Unpack(a[3]);
  long long ks, vs;
  if (dtype_code(k) < 0 || v.scalar_type() != k.scalar_type() || !rows_of(k, keys->device(), c->heads, c->head_dim, ks) ||
      !rows_of(v, keys->device(), c->heads, c->head_dim, vs) || k.size(0) != v.size(0) || (a[7] == Py_None) != (a[8] == Py_None))
    Py_RETURN_NONE;
  long long tokens = k.size(0);
  const int *rows = nullptr, *row_offsets = nullptr;
  if (a[7] != Py_None) {
    if (!THPVariable_Check(a[7]) || !THPVariable_Check(a[8])) Py_RETURN_NONE;
    const at::Tensor &r = THPVariable_Unpack(a[7]), &ro = THPVariable_Unpack(a[8]);
    tokens = r.numel();
    if (!is_int(tokens) || !fits(r, at::kInt, keys->device(), 1) || !fits(ro, at::kInt, keys->device(), t.batch + 1ll)) Py_RETURN_NONE;
    rows = static_cast<const int*>(r.data_ptr());
    row_offsets = static_cast<const int*>(ro.data_ptr());
  }
  return PyLong_FromLong(call(g_write, c, &t, dtype_code(k), (int)tokens, k.data_ptr(), v.data_ptr(), ks, vs, rows, row_offsets, (int)k.size(0),
                              current_stream()));
  END_HANDLE_TH_ERRORS
}

// cache_read(cache, keys, offsets, lengths, table, n, any tensor of the type wanted or None) -> (k, v), or the library's status; None
// where an argument is not of the usual kind.
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const covspec_cache* c;
  const at::Tensor* keys;
  covspec_tokens t;
  long long tokens;
  if (n != 7 || !cache_of(a[0], a[1], c, keys) || !tokens_of(a + 2, keys->device(), t) || !PyLong_CheckExact(a[5]) || !PyLong_CheckExact(a[6])) Py_RETURN_NONE;
  if (!int_arg(a[5], tokens)) return nullptr;
  const long dtype = PyLong_AsLong(a[6]);
  if (!is_int(tokens) || tokens < 0 || dtype < 0 || dtype > 2) Py_RETURN_NONE;
  const auto options = keys->options().dtype(dtype == 0 ? at::kFloat : dtype == 1 ? at::kBFloat16 : at::kHalf);
  at::Tensor k = at::empty({tokens, c->heads, c->head_dim}, options), v = at::empty({tokens, c->heads, c->head_dim}, options);
  const int st = call(g_read, c, &t, (int)dtype, (int)tokens, k.data_ptr(), v.data_ptr(), current_stream());
  if (st) return PyLong_FromLong(st);
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(k)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(v)));
  return out;
  END_HANDLE_TH_ERRORS
}

// cache_attend(cache, keys, workspace bytes, q, offsets, lengths, table, scale, window, max_new, lse wanted, out or None) -> out or
// (out, lse), or the library's status; None where an argument is not of the usual kind.
PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const covspec_cache* c;
  const at::Tensor* keys;
  covspec_tokens t;
  if (n != 12 || !cache_of(a[0], a[1], c, keys) || !THPVariable_Check(a[3]) || !tokens_of(a + 4, keys->device(), t)) Py_RETURN_NONE;
  const at::Tensor& q = THPVariable_Unpack(a[3]);
  long long qs, os, size, window, most;
  if (dtype_code(q) < 1 || q.dim() != 3 || !is_int(q.size(1)) || !rows_of(q, keys->device(), q.size(1), c->head_dim, qs)) Py_RETURN_NONE;
  const double scale = PyFloat_AsDouble(a[7]);
  if (scale == -1.0 && PyErr_Occurred()) return nullptr;
  if (!int_arg(a[2], size) || !int_arg(a[8], window) || !int_arg(a[9], most)) return nullptr;
  if (!is_int(window) || !is_int(most)) Py_RETURN_NONE;
  const int logs = PyObject_IsTrue(a[10]);
  if (logs < 0) return nullptr;
  at::Tensor out;
  if (a[11] == Py_None) {
    out = at::empty({q.size(0), q.size(1), q.size(2)}, q.options());
  } else {
    if (!THPVariable_Check(a[11])) Py_RETURN_NONE;
    out = THPVariable_Unpack(a[11]);
    if (out.scalar_type() != q.scalar_type()) Py_RETURN_NONE;
  }
  if (!rows_of(out, keys->device(), q.size(1), c->head_dim, os) || out.size(0) < q.size(0)) Py_RETURN_NONE;
  at::Tensor lse;
  if (logs) lse = at::empty({q.size(0), q.size(1)}, q.options().dtype(at::kFloat));
  // from torch's pool, like the outputs: it knows streams and captures, so no two calls in flight share it
  at::Tensor work = at::empty({size}, q.options().dtype(at::kByte));
  const int st = call(g_attend, c, &t, dtype_code(q), (int)q.size(0), q.data_ptr(), qs, (int)q.size(1), (float)scale, (int)window, (int)most,
                      out.data_ptr(), os, logs ? static_cast<float*>(lse.data_ptr()) : nullptr, work.data_ptr(), size, current_stream());
  if (st) return PyLong_FromLong(st);
  if (!logs) return THPVariable_Wrap(std::move(out));
  PyObject* both = PyTuple_New(2);
  if (!both) return nullptr;
  PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(std::move(out)));
  PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(std::move(lse)));
  return both;
  END_HANDLE_TH_ERRORS
}

// edit_logits(z, row_offsets, history, history_offsets, prompt_lengths, drafted, repetition, presence, frequency, bias_ids,
// bias_values, bias_offsets, mask, vocab, out; all but the first two may be None) -> out, or the library's status; None where an
// argument is not of the usual kind.
PyObject* edit_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15 || !THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) Py_RETURN_NONE;
  for (int i = 2; i < 15; ++i)
    if (i != 13 && a[i] != Py_None && !THPVariable_Check(a[i])) Py_RETURN_NONE;
  const at::Tensor &z = THPVariable_Unpack(a[0]), &offsets = THPVariable_Unpack(a[1]);
  if (!on_current_device(z) || z.dim() != 2 || !z.is_contiguous() || dtype_code(z) < 0 || !is_int(z.size(0))) Py_RETURN_NONE;
  const auto dev = z.device();
  const long long rows = z.size(0), ld = z.size(1), batch = offsets.numel() - 1;
  if (batch < 1 || !is_int(batch) || !fits(offsets, at::kInt, dev, batch + 1)) Py_RETURN_NONE;
  long long vocab = ld;
  if (a[13] != Py_None && !int_arg(a[13], vocab)) return nullptr;
  if (!is_int(vocab) || vocab < 1) Py_RETURN_NONE;
  if ((a[2] == Py_None) != (a[3] == Py_None) || (a[9] == Py_None) != (a[10] == Py_None) || (a[9] == Py_None) != (a[11] == Py_None)) Py_RETURN_NONE;
  const long long hist = a[2] == Py_None ? 0 : THPVariable_Unpack(a[2]).numel(), bias = a[9] == Py_None ? 0 : THPVariable_Unpack(a[9]).numel();
  if (!is_int(hist) || !is_int(bias)) Py_RETURN_NONE;
  const long long least[13] = {0, 0, 0, batch + 1, batch, rows, batch, batch, batch, 0, bias, batch + 1, 0};
  const void* at_[13] = {};
  for (int i = 2; i < 12; ++i) {
    if (a[i] == Py_None) continue;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (!fits(t, (i >= 6 && i <= 8) || i == 10 ? at::kFloat : at::kInt, dev, least[i])) Py_RETURN_NONE;
    at_[i] = t.data_ptr();
  }
  auto ints = [&](int i) { return static_cast<const int*>(at_[i]); };
  auto floats = [&](int i) { return static_cast<const float*>(at_[i]); };
  covspec_edits e{(int)batch, static_cast<const int*>(offsets.data_ptr()), ints(2), ints(3), (int)hist, ints(4), ints(5), floats(6), floats(7),
                  floats(8), ints(9), floats(10), ints(11), (int)bias, nullptr, 0};
  if (a[12] != Py_None) {
    const at::Tensor& m = THPVariable_Unpack(a[12]);
    if (m.dim() != 2 || m.size(0) < rows || m.size(1) < (vocab + 31) / 32 || !fits(m, at::kInt, dev, 0)) Py_RETURN_NONE;
    e.mask = m.data_ptr();
    e.mask_stride = 4 * m.size(1);
  }
  at::Tensor out;
  if (a[14] == Py_None) {
    out = at::empty({rows, ld}, z.options());
  } else {
    out = THPVariable_Unpack(a[14]);
    if (!out.sizes().equals(z.sizes()) || !fits(out, z.scalar_type(), dev, z.numel())) Py_RETURN_NONE;
  }
  const int st = call(g_edit, dtype_code(z), (int)rows, (int)vocab, ld, z.data_ptr(), out.data_ptr(), &e, current_stream());
  if (st) return PyLong_FromLong(st);
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"correct", (PyCFunction)(void (*)(void))correct, METH_FASTCALL, nullptr},
                         {"candidates", (PyCFunction)(void (*)(void))candidates, METH_FASTCALL, nullptr},
                         {"static_score", (PyCFunction)(void (*)(void))static_score, METH_FASTCALL, nullptr},
                         {"cache_write", (PyCFunction)(void (*)(void))cache_write, METH_FASTCALL, nullptr},
                         {"cache_read", (PyCFunction)(void (*)(void))cache_read, METH_FASTCALL, nullptr},
                         {"cache_attend", (PyCFunction)(void (*)(void))cache_attend, METH_FASTCALL, nullptr},
                         {"edit_logits", (PyCFunction)(void (*)(void))edit_logits, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module_def); }
