// The calls of a decode loop, from Python in native code: rdkv_decode_attn and rdkv_cache_append, and rdkv_slots_append,
// rdkv_slots_decode_attn, rdkv_slots_read, rdkv_slots_fill, rdkv_slots_tree_attn and rdkv_slots_accept; and
// rdkv_prompt_attn_bf16.
//
// A decode step of a short context takes the GPU 5.2 us.  Through ctypes it took the host 7.4: 3.6 in the call itself, 2.5 for
// two result tensors made from Python and the rest for converting arguments one by one.  Here the tensors are unpacked and
// made by PyTorch's C++ interface: 5.8 us per step (4K keys, 2 KV heads), a request of 32K keys and 64 tokens with results
// given 1054 -> 988 us.  What is not a plain tensor call (an argument that is no tensor, one of a subclass, one that is not
// contiguous) is left to the ctypes path, which says what is wrong with it: the functions then return None.  (On slot
// caches, host us with results made: append 6.8 -> 4.3, step 9.3 -> 6.5, read 8.7 -> 5.3, a fill of four launches 19.7 -> 14.4.  The GPU
// takes 4.6 for an append to 2 items of 1000 slots, 3.0 for a read of a few rows.  Trees 12.1 -> 8.2 of 13, accepting 15.3 -> 10.0 of 15,
// prompts 14.0 -> 7.5 of 10.4 for 600 tokens.)
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <cstdint>
#include <vector>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include "rdkv.h"

namespace {

decltype(&rdkv_decode_attn) g_decode = nullptr;
decltype(&rdkv_cache_append) g_append = nullptr;
decltype(&rdkv_slots_append) g_slots_append = nullptr;
decltype(&rdkv_slots_decode_attn) g_slots_decode = nullptr;
decltype(&rdkv_slots_read) g_slots_read = nullptr;
decltype(&rdkv_slots_fill) g_slots_fill = nullptr;
decltype(&rdkv_slots_fill_workspace_bytes) g_slots_fill_bytes = nullptr;
decltype(&rdkv_slots_tree_attn) g_slots_tree = nullptr;
decltype(&rdkv_slots_tree_workspace_bytes) g_slots_tree_bytes = nullptr;
decltype(&rdkv_prompt_attn_bf16) g_prompt = nullptr;
decltype(&rdkv_slots_accept) g_slots_accept = nullptr;
decltype(&rdkv_slots_accept_workspace_bytes) g_slots_accept_bytes = nullptr;

// a contiguous tensor's memory
bool pointer(PyObject* o, void** p) {
  if (!THPVariable_CheckExact(o)) return false;      // (a subclass has methods of its own)
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_contiguous()) return false;
  *p = t.data_ptr();
  return true;
}

// a cache's handle: a number, None, or a ctypes pointer
bool handle(PyObject* o, long long* h) {
  if (o == Py_None) {
    *h = 0;
    return true;
  }
  if (PyLong_Check(o)) {
    *h = PyLong_AsLongLong(o);
    return !PyErr_Occurred();
  }
  static PyObject* const name = PyUnicode_InternFromString("value");
  PyObject* v = PyObject_GetAttr(o, name);
  if (!v) return false;
  const bool ok = v == Py_None || PyLong_Check(v);
  *h = v == Py_None || !ok ? 0 : PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (!ok) PyErr_SetString(PyExc_TypeError, "not a handle");
  return ok && !PyErr_Occurred();
}

bool integers(PyObject* const* args, int n, long long* out) {
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(args[i]);
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// bind(address of rdkv_decode_attn, address of rdkv_cache_append)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  long long a[2];
  if (n != 2 || !integers(args, 2, a)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind takes two addresses");
    return nullptr;
  }
  g_decode = reinterpret_cast<decltype(g_decode)>(a[0]);
  g_append = reinterpret_cast<decltype(g_append)>(a[1]);
  Py_RETURN_NONE;
}

// decode(cache, stream, batch, hq, d, q, out or None, lse or None) -> (status, out, lse) or None
PyObject* decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long long h, a[4];
  if (n != 8 || !handle(args[0], &h) || !integers(args + 1, 4, a)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "decode takes eight arguments");
    return nullptr;
  }
  void *q, *out = nullptr, *lse = nullptr;
  if (!g_decode || !pointer(args[5], &q)) Py_RETURN_NONE;
  const bool make_out = args[6] == Py_None, make_lse = args[7] == Py_None;
  if ((!make_out && !pointer(args[6], &out)) || (!make_lse && !pointer(args[7], &lse))) Py_RETURN_NONE;
  at::Tensor new_out, new_lse;
  const auto options = at::TensorOptions().dtype(at::kFloat).device(THPVariable_Unpack(args[5]).device());
  if (make_out) {
    new_out = at::empty({a[1], a[2], a[3]}, options);
    out = new_out.data_ptr();
  }
  if (make_lse) {
    new_lse = at::empty({a[1], a[2]}, options);
    lse = new_lse.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_decode(reinterpret_cast<rdkv_cache*>(h), q, static_cast<float*>(out), static_cast<float*>(lse), reinterpret_cast<void*>(a[0]));
  Py_END_ALLOW_THREADS
  THPObjectPtr py_out(make_out ? THPVariable_Wrap(std::move(new_out)) : Py_NewRef(args[6]));
  THPObjectPtr py_lse(make_lse ? THPVariable_Wrap(std::move(new_lse)) : Py_NewRef(args[7]));
  if (!py_out || !py_lse) return nullptr;
  return Py_BuildValue("(iNN)", status, py_out.release(), py_lse.release());
  END_HANDLE_TH_ERRORS
}

// append(cache, stream, k_new, v_new) -> status or None
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long long h, stream;
  if (n != 4 || !handle(args[0], &h) || !integers(args + 1, 1, &stream)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "append takes four arguments");
    return nullptr;
  }
  void *k, *v;
  if (!g_append || !pointer(args[2], &k) || !pointer(args[3], &v)) Py_RETURN_NONE;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_append(reinterpret_cast<rdkv_cache*>(h), k, v, reinterpret_cast<void*>(stream));
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}

// bind_slots(addresses of rdkv_slots_append, rdkv_slots_decode_attn, rdkv_slots_read, rdkv_slots_fill, rdkv_slots_fill_workspace_bytes)
PyObject* bind_slots(PyObject*, PyObject* const* args, Py_ssize_t n) {
  long long a[5];
  if (n != 5 || !integers(args, 5, a)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind_slots takes five addresses");
    return nullptr;
  }
  g_slots_append = reinterpret_cast<decltype(g_slots_append)>(a[0]);
  g_slots_decode = reinterpret_cast<decltype(g_slots_decode)>(a[1]);
  g_slots_read = reinterpret_cast<decltype(g_slots_read)>(a[2]);
  g_slots_fill = reinterpret_cast<decltype(g_slots_fill)>(a[3]);
  g_slots_fill_bytes = reinterpret_cast<decltype(g_slots_fill_bytes)>(a[4]);
  Py_RETURN_NONE;
}

// bind_tree(addresses of rdkv_slots_tree_attn, rdkv_slots_tree_workspace_bytes, rdkv_slots_accept, rdkv_slots_accept_workspace_bytes,
//           rdkv_prompt_attn_bf16)
PyObject* bind_tree(PyObject*, PyObject* const* args, Py_ssize_t n) {
  long long a[5];
  if (n != 5 || !integers(args, 5, a)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind_tree takes five addresses");
    return nullptr;
  }
  g_slots_tree = reinterpret_cast<decltype(g_slots_tree)>(a[0]);
  g_slots_tree_bytes = reinterpret_cast<decltype(g_slots_tree_bytes)>(a[1]);
  g_slots_accept = reinterpret_cast<decltype(g_slots_accept)>(a[2]);
  g_slots_accept_bytes = reinterpret_cast<decltype(g_slots_accept_bytes)>(a[3]);
  g_prompt = reinterpret_cast<decltype(g_prompt)>(a[4]);
  Py_RETURN_NONE;
}

// What the calls on a slot cache begin with: (address of its struct, stream, index of its device, ..)
struct SlotsCall {
  const rdkv_slots* s;
  void* stream;
  int device;
  bool ok;
  SlotsCall(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : ok(false) {
    long long a[3];
    if (n != want || !integers(args, 3, a)) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "a call on a slot cache takes other arguments");
      return;
    }
    s = reinterpret_cast<const rdkv_slots*>(a[0]);
    stream = reinterpret_cast<void*>(a[1]);
    device = static_cast<int>(a[2]);
    ok = true;
  }
  at::TensorOptions options(at::ScalarType type) const { return at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<at::DeviceIndex>(device)); }
  // a contiguous tensor of this type and shape on the cache's device: its memory
  bool plain(PyObject* o, at::ScalarType type, at::IntArrayRef shape, void** p) const {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.device().index() != device || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous()) return false;
    *p = t.data_ptr();
    return true;
  }
};
// a result: the tensor given (o) or made
PyObject* result(at::Tensor&& made, PyObject* o) { return made.defined() ? THPVariable_Wrap(std::move(made)) : Py_NewRef(o); }

// slots_append(.., k_new, v_new, slot or None) -> (status, slot) or None
PyObject* slots_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n, 6);
  if (!c.ok) return nullptr;
  void *k, *v, *slot;
  const int64_t row[3] = {c.s->batch, c.s->hkv, c.s->head_dim};
  const at::IntArrayRef rows(row, 3), items(row, 2);
  if (!g_slots_append || !c.plain(args[3], at::kBFloat16, rows, &k) || !c.plain(args[4], at::kBFloat16, rows, &v)) Py_RETURN_NONE;
  at::Tensor made;
  if (args[5] == Py_None) {
    made = at::empty(items, c.options(at::kInt));
    slot = made.data_ptr();
  } else if (!c.plain(args[5], at::kInt, items, &slot)) {
    Py_RETURN_NONE;
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_append(c.s, k, v, static_cast<int32_t*>(slot), c.stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr out(result(std::move(made), args[5]));
  return out ? Py_BuildValue("(iN)", status, out.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

// slots_decode(.., q, out or None, lse or None, workspace or None, bytes of a workspace) -> (status, out, lse) or None
PyObject* slots_decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n, 8);
  long long bytes;
  if (!c.ok || !integers(args + 7, 1, &bytes)) return nullptr;
  void *q, *out, *lse, *ws;
  const int64_t row[3] = {c.s->batch, c.s->hq, c.s->head_dim};
  const at::IntArrayRef rows(row, 3), heads(row, 2);
  if (!g_slots_decode || !c.plain(args[3], at::kBFloat16, rows, &q)) Py_RETURN_NONE;
  at::Tensor new_out, new_lse, new_ws;
  const bool make_out = args[4] == Py_None, make_lse = args[5] == Py_None, make_ws = args[6] == Py_None;
  if ((!make_out && !c.plain(args[4], at::kFloat, rows, &out)) || (!make_lse && !c.plain(args[5], at::kFloat, heads, &lse))) Py_RETURN_NONE;
  if (!make_ws) {
    if (!THPVariable_CheckExact(args[6])) Py_RETURN_NONE;
    bytes = THPVariable_Unpack(args[6]).numel();
    if (!c.plain(args[6], at::kByte, THPVariable_Unpack(args[6]).sizes(), &ws)) Py_RETURN_NONE;
  } else {
    new_ws = at::empty({std::max<int64_t>(bytes, 16)}, c.options(at::kByte));
    ws = new_ws.data_ptr();
  }
  if (make_out) {
    new_out = at::empty(rows, c.options(at::kFloat));
    out = new_out.data_ptr();
  }
  if (make_lse) {
    new_lse = at::empty(heads, c.options(at::kFloat));
    lse = new_lse.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_decode(c.s, q, static_cast<float*>(out), static_cast<float*>(lse), ws, static_cast<size_t>(bytes), c.stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr py_out(result(std::move(new_out), args[4])), py_lse(result(std::move(new_lse), args[5]));
  return py_out && py_lse ? Py_BuildValue("(iNN)", status, py_out.release(), py_lse.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

// slots_read(.., index or None, n or None, K or None, V or None) -> (status, K, V) or None
PyObject* slots_read(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n_args, 7);
  if (!c.ok) return nullptr;
  long long n = c.s->capacity;
  void *index = nullptr, *k, *v;
  if (args[3] != Py_None) {
    if (!THPVariable_CheckExact(args[3])) Py_RETURN_NONE;
    const at::Tensor& t = THPVariable_Unpack(args[3]);
    if (t.dim() != 3) Py_RETURN_NONE;
    n = t.size(2);
  }
  if (args[4] != Py_None) {
    long long given;
    if (!PyLong_CheckExact(args[4])) Py_RETURN_NONE;
    int over;
    given = PyLong_AsLongLongAndOverflow(args[4], &over);
    if (over || given < 0 || given > INT32_MAX || (args[3] != Py_None && given != n)) Py_RETURN_NONE;
    n = given;
  }
  const int64_t row[4] = {c.s->batch, c.s->hkv, n, c.s->head_dim};
  const at::IntArrayRef rows(row, 4);
  if (!g_slots_read || n > INT32_MAX || (args[3] != Py_None && !c.plain(args[3], at::kInt, at::IntArrayRef(row, 3), &index))) Py_RETURN_NONE;
  at::Tensor new_k, new_v;
  const bool make_k = args[5] == Py_None, make_v = args[6] == Py_None;
  if ((!make_k && !c.plain(args[5], at::kBFloat16, rows, &k)) || (!make_v && !c.plain(args[6], at::kBFloat16, rows, &v))) Py_RETURN_NONE;
  if (make_k) {
    new_k = at::empty(rows, c.options(at::kBFloat16));
    k = new_k.data_ptr();
  }
  if (make_v) {
    new_v = at::empty(rows, c.options(at::kBFloat16));
    v = new_v.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_read(c.s, static_cast<const int32_t*>(index), static_cast<int32_t>(n), k, v, c.stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr py_k(result(std::move(new_k), args[5])), py_v(result(std::move(new_v), args[6]));
  return py_k && py_v ? Py_BuildValue("(iNN)", status, py_k.release(), py_v.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

// a whole number of 32 bits
bool number(PyObject* o, int32_t* x) {
  int over = 0;
  const long long v = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &over) : -1 - static_cast<long long>(INT32_MAX) - 1;
  *x = static_cast<int32_t>(v);
  return over == 0 && v >= INT32_MIN && v <= INT32_MAX;
}

// slots_fill(.., K, V, seq_lens, w_tok or None, first) -> status or None
PyObject* slots_fill(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n_args, 8);
  if (!c.ok) return nullptr;
  if (!g_slots_fill || !g_slots_fill_bytes || !PyList_CheckExact(args[5]) || !PyLong_CheckExact(args[7])) Py_RETURN_NONE;
  const Py_ssize_t n = PyList_GET_SIZE(args[5]);
  int32_t first;
  if (n > INT32_MAX || !number(args[7], &first)) Py_RETURN_NONE;
  std::vector<int32_t> lens(n + 1);
  int64_t rows = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!number(PyList_GET_ITEM(args[5], i), &lens[i])) Py_RETURN_NONE;
    rows += std::max(lens[i], 0);
  }
  rows *= c.s->hkv;
  // ragged: any shape of as many numbers
  const auto ragged = [&](PyObject* o, at::ScalarType type, int64_t numbers, void** p) {
    return THPVariable_CheckExact(o) && THPVariable_Unpack(o).numel() == numbers && c.plain(o, type, THPVariable_Unpack(o).sizes(), p);
  };
  void *k, *v, *w = nullptr;
  if (!ragged(args[3], at::kBFloat16, rows * c.s->head_dim, &k) || !ragged(args[4], at::kBFloat16, rows * c.s->head_dim, &v)) Py_RETURN_NONE;
  if (args[6] != Py_None && !ragged(args[6], at::kFloat, rows, &w)) Py_RETURN_NONE;
  const size_t bytes = g_slots_fill_bytes(c.s, static_cast<int32_t>(n), lens.data());
  at::Tensor ws;
  if (bytes > 0) ws = at::empty({static_cast<int64_t>(bytes)}, c.options(at::kByte));
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_fill(c.s, first, static_cast<int32_t>(n), lens.data(), k, v, static_cast<const float*>(w), bytes > 0 ? ws.data_ptr() : nullptr, bytes, c.stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
  END_HANDLE_TH_ERRORS
}

// prompt(stream, index of the device, Q, K, V, seq_lens, hq, hkv, head_dim, window, sinks, score_cap, slopes or None, out or None, lse or None)
//   -> (status, out, lse) or None
PyObject* prompt(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  long long a[2];
  if (n_args != 15 || !integers(args, 2, a)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "prompt takes fifteen arguments");
    return nullptr;
  }
  void* stream = reinterpret_cast<void*>(a[0]);
  const auto device = static_cast<at::DeviceIndex>(a[1]);
  rdkv_prompt c = {};
  if (!g_prompt || !PyList_CheckExact(args[5]) || !number(args[6], &c.hq) || !number(args[7], &c.hkv) || !number(args[8], &c.head_dim) ||
      !number(args[9], &c.window) || !number(args[10], &c.sinks) || !(PyFloat_CheckExact(args[11]) || PyLong_CheckExact(args[11])))
    Py_RETURN_NONE;
  const Py_ssize_t n = PyList_GET_SIZE(args[5]);
  if (n > INT32_MAX || c.hq < 1 || c.hkv < 1 || c.head_dim < 1) Py_RETURN_NONE;
  std::vector<int32_t> lens(n + 1);
  int64_t tokens = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!number(PyList_GET_ITEM(args[5], i), &lens[i])) Py_RETURN_NONE;
    tokens += std::max(lens[i], 0);
  }
  constexpr int32_t kMany = 65536;                 // (so that no product of sizes overflows)
  if (tokens > INT32_MAX || c.hq > kMany || c.hkv > kMany || c.head_dim > kMany) Py_RETURN_NONE;
  c.batch = static_cast<int32_t>(n);
  c.seq_lens = lens.data();
  const double cap = PyFloat_AsDouble(args[11]);
  if (cap == -1.0 && PyErr_Occurred()) return nullptr;
  c.score_cap = static_cast<float>(cap);
  if (c.score_cap == 0.f && cap != 0.0) Py_RETURN_NONE;
  // flat rows, or [tokens, heads, head_dim] of rows whose heads lie side by side, none of which overlap
  const auto rows = [&](PyObject* o, int64_t heads, int64_t* stride, void** p) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.device().index() != device || t.scalar_type() != at::kBFloat16) return false;
    const int64_t d = c.head_dim;
    *p = t.data_ptr();
    *stride = 0;
    if (t.dim() == 1 || t.dim() == 2) return t.is_contiguous() && t.numel() == tokens * heads * d && (t.dim() == 1 || t.size(1) == d);
    if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != heads || t.size(2) != d) return false;
    *stride = tokens > 1 ? t.stride(0) : heads * d;
    return tokens == 0 || (*stride >= heads * d && t.stride(2) == 1 && (heads == 1 || t.stride(1) == d));
  };
  void *q, *k, *v, *out, *lse, *slopes = nullptr;
  if (!rows(args[2], c.hq, &c.q_stride, &q) || !rows(args[3], c.hkv, &c.k_stride, &k) || !rows(args[4], c.hkv, &c.v_stride, &v)) Py_RETURN_NONE;
  const auto plain = [&](PyObject* o, int64_t numbers, void** p) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    *p = t.data_ptr();
    return t.is_cuda() && t.device().index() == device && t.scalar_type() == at::kFloat && t.is_contiguous() && t.numel() == numbers;
  };
  if (args[12] != Py_None && (!plain(args[12], c.hq, &slopes) || THPVariable_Unpack(args[12]).dim() != 1)) Py_RETURN_NONE;
  c.slopes = static_cast<const float*>(slopes);
  if ((args[13] != Py_None && !rows(args[13], c.hq, &c.out_stride, &out)) || (args[14] != Py_None && !plain(args[14], tokens * c.hq, &lse))) Py_RETURN_NONE;
  const auto options = at::TensorOptions().device(at::kCUDA, device);
  at::Tensor new_out, new_lse;
  if (args[13] == Py_None) {
    const at::Tensor& t = THPVariable_Unpack(args[2]);
    new_out = at::empty(t.sizes(), options.dtype(at::kBFloat16));
    out = new_out.data_ptr();
    c.out_stride = t.dim() == 3 ? static_cast<int64_t>(c.hq) * c.head_dim : 0;
  }
  if (args[14] == Py_None) {
    new_lse = at::empty({tokens * c.hq}, options.dtype(at::kFloat));
    lse = new_lse.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_prompt(&c, q, k, v, out, static_cast<float*>(lse), stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr py_out(result(std::move(new_out), args[13])), py_lse(result(std::move(new_lse), args[14]));
  return py_out && py_lse ? Py_BuildValue("(iNN)", status, py_out.release(), py_lse.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

// The drafted tokens of a tree: q (or None), k_draft, v_draft; n of them a sequence
struct Drafted {
  void *q = nullptr, *k, *v;
  int64_t n = 0;
  bool ok = false;
  Drafted(const SlotsCall& c, PyObject* const* args) {
    if (!THPVariable_CheckExact(args[1])) return;
    const at::Tensor& t = THPVariable_Unpack(args[1]);
    if (t.dim() != 4 || t.size(1) > INT32_MAX) return;
    n = t.size(1);
    const int64_t row[4] = {c.s->batch, n, c.s->hkv, c.s->head_dim}, q_row[4] = {row[0], n, c.s->hq, row[3]};
    ok = (args[0] == Py_None || c.plain(args[0], at::kBFloat16, at::IntArrayRef(q_row, 4), &q)) &&
         c.plain(args[1], at::kBFloat16, at::IntArrayRef(row, 4), &k) && c.plain(args[2], at::kBFloat16, at::IntArrayRef(row, 4), &v);
  }
};
// a workspace: the tensor given, or a new one of so many bytes (`made`)
bool workspace(const SlotsCall& c, PyObject* o, size_t* bytes, void** p, at::Tensor* made) {
  if (o == Py_None) {
    *made = at::empty({std::max<int64_t>(static_cast<int64_t>(*bytes), 16)}, c.options(at::kByte));
    *p = made->data_ptr();
    return true;
  }
  if (!THPVariable_CheckExact(o)) return false;
  *bytes = static_cast<size_t>(THPVariable_Unpack(o).numel());
  return c.plain(o, at::kByte, THPVariable_Unpack(o).sizes(), p);
}

// slots_tree(.., q, k_draft, v_draft, parent, counts or None, out or None, stats or None, workspace or None) -> (status, out, stats) or None
PyObject* slots_tree(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n_args, 11);
  if (!c.ok) return nullptr;
  const Drafted d(c, args + 3);
  if (!g_slots_tree || !g_slots_tree_bytes || !d.ok || !d.q) Py_RETURN_NONE;
  const int64_t batch = c.s->batch, row[4] = {batch, d.n, c.s->hq, c.s->head_dim}, stat[4] = {batch, d.n, c.s->hq, 2}, tokens[2] = {batch, d.n};
  const at::IntArrayRef rows(row, 4), pairs(stat, 4);
  void *parent, *counts = nullptr, *out, *stats, *ws;
  if (!c.plain(args[6], at::kInt, at::IntArrayRef(tokens, 2), &parent) ||
      (args[7] != Py_None && !c.plain(args[7], at::kInt, at::IntArrayRef(tokens, 1), &counts)) ||
      (args[8] != Py_None && !c.plain(args[8], at::kBFloat16, rows, &out)) || (args[9] != Py_None && !c.plain(args[9], at::kFloat, pairs, &stats)))
    Py_RETURN_NONE;
  size_t bytes = g_slots_tree_bytes(c.s, static_cast<int32_t>(d.n));
  at::Tensor new_out, new_stats, new_ws;
  if (!workspace(c, args[10], &bytes, &ws, &new_ws)) Py_RETURN_NONE;
  if (args[8] == Py_None) {
    new_out = at::empty(rows, c.options(at::kBFloat16));
    out = new_out.data_ptr();
  }
  if (args[9] == Py_None) {
    new_stats = at::empty(pairs, c.options(at::kFloat));
    stats = new_stats.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_tree(c.s, static_cast<int32_t>(d.n), d.q, d.k, d.v, static_cast<const int32_t*>(parent), static_cast<const int32_t*>(counts), out,
                        static_cast<float*>(stats), ws, bytes, c.stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr py_out(result(std::move(new_out), args[8])), py_stats(result(std::move(new_stats), args[9]));
  return py_out && py_stats ? Py_BuildValue("(iNN)", status, py_out.release(), py_stats.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

// slots_accept(.., q or None, k_draft, v_draft, path, stats or None, slot or None, workspace or None) -> (status, slot) or None
PyObject* slots_accept(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  const SlotsCall c(args, n_args, 10);
  if (!c.ok) return nullptr;
  const Drafted d(c, args + 3);
  if (!g_slots_accept || !g_slots_accept_bytes || !d.ok || !THPVariable_CheckExact(args[6])) Py_RETURN_NONE;
  const at::Tensor& t = THPVariable_Unpack(args[6]);
  if (t.dim() != 2 || t.size(1) > INT32_MAX) Py_RETURN_NONE;
  const int64_t batch = c.s->batch, m = t.size(1), tokens[2] = {batch, m}, stat[4] = {batch, d.n, c.s->hq, 2}, taken[3] = {batch, c.s->hkv, m};
  const at::IntArrayRef slots(taken, 3);
  void *path, *stats = nullptr, *slot, *ws;
  if (!c.plain(args[6], at::kInt, at::IntArrayRef(tokens, 2), &path) ||
      (args[7] != Py_None && !c.plain(args[7], at::kFloat, at::IntArrayRef(stat, 4), &stats)) || (args[8] != Py_None && !c.plain(args[8], at::kInt, slots, &slot)))
    Py_RETURN_NONE;
  size_t bytes = g_slots_accept_bytes(c.s);
  at::Tensor made, new_ws;
  if (!workspace(c, args[9], &bytes, &ws, &new_ws)) Py_RETURN_NONE;
  if (args[8] == Py_None) {
    made = at::empty(slots, c.options(at::kInt));
    slot = made.data_ptr();
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = g_slots_accept(c.s, static_cast<int32_t>(d.n), static_cast<int32_t>(m), d.q, d.k, d.v, static_cast<const int32_t*>(path), static_cast<const float*>(stats),
                          static_cast<int32_t*>(slot), ws, bytes, c.stream);
  Py_END_ALLOW_THREADS
  THPObjectPtr out(result(std::move(made), args[8]));
  return out ? Py_BuildValue("(iN)", status, out.release()) : nullptr;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
    {"bind_slots", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind_slots)), METH_FASTCALL, nullptr},
    {"slots_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_append)), METH_FASTCALL, nullptr},
    {"slots_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_decode)), METH_FASTCALL, nullptr},
    {"slots_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_read)), METH_FASTCALL, nullptr},
    {"slots_fill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_fill)), METH_FASTCALL, nullptr},
    {"bind_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind_tree)), METH_FASTCALL, nullptr},
    {"prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prompt)), METH_FASTCALL, nullptr},
    {"slots_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_tree)), METH_FASTCALL, nullptr},
    {"slots_accept", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(slots_accept)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rdkv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rdkv_call() { return PyModule_Create(&module); }
