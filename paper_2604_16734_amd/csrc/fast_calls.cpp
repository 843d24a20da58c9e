// The per-layer calls of Cache (binding.py) and those of pages.py from Python without ctypes: functions that look at the tensors and
// call the C entry point.  A decode step of a small cache takes the GPU less than the checks and conversions of the same call took
// in Python.
//
// call(entry, handle, layer, tensors, q_row, kv_row, device, stream, token_begin) -> the entry point's code, or None where anything
// about the arguments is not plainly as it should be: the caller then takes its Python path, which has the same checks and says what is
// wrong.  page_rows, paged_decode and prompt (below) likewise.  Nothing is kept from one call to the next, and no C++ exception leaves: what a tensor throws when it is looked at counts as not plain.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "kvp.h"

// where the tensors have to be (the tests build the module for the CPU, too)
#ifndef KVP_TENSOR_DEVICE
#define KVP_TENSOR_DEVICE c10::DeviceType::CUDA
#endif

namespace {

constexpr int kMostTensors = 5;

// a plain tensor of `device` and of this type; its address is then what data_ptr() gives
bool plain_of(PyObject* o, int64_t device, at::ScalarType type, const at::Tensor** out) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.is_nested()) return false;
  const auto keys = t.key_set();
  if (keys.has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                        c10::DispatchKey::Functionalize, c10::DispatchKey::Batched, c10::DispatchKey::ZeroTensor})))
    return false;
  if (t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != type) return false;
  const c10::Device d = t.device();
  if (d.type() != KVP_TENSOR_DEVICE || d.index() != device) return false;
  *out = &t;
  return true;
}
// a contiguous one of bf16
bool plain(PyObject* o, int64_t device, const at::Tensor** out) { return plain_of(o, device, at::kBFloat16, out) && (*out)->is_contiguous(); }

bool small_int(PyObject* o, int32_t* out) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow || v < INT32_MIN || v > INT32_MAX) return false;
  *out = (int32_t)v;
  return true;
}

bool address(PyObject* o, void** out) {
  if (!PyLong_CheckExact(o)) return false;
  const unsigned long long v = PyLong_AsUnsignedLongLong(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *out = (void*)(uintptr_t)v;
  return true;
}

bool pair(PyObject* o, int64_t (&out)[2]) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) return false;
  for (int i = 0; i < 2; ++i) {
    int32_t v;
    if (!small_int(PyTuple_GET_ITEM(o, i), &v)) return false;
    out[i] = v;
  }
  return true;
}

bool rows_of(const at::Tensor& t, const int64_t (&row)[2], int64_t rows) {       // [rows, row[0], row[1]]
  return t.dim() == 3 && t.size(0) == rows && t.size(1) == row[0] && t.size(2) == row[1];
}

// the tensors' addresses, the rows of K and those of q_obs, where all are plain and of the shapes that belong together
bool plain_tensors(PyObject* list, Py_ssize_t n_tensors, bool step, const int64_t (&q_row)[2], const int64_t (&kv_row)[2], int64_t device,
                   void* (&p)[kMostTensors], int64_t* rows, int64_t* n_obs) {
  const at::Tensor* t[kMostTensors];
  for (Py_ssize_t i = 0; i < n_tensors; ++i) {
    if (!plain(PyTuple_GET_ITEM(list, i), device, &t[i])) return false;
    p[i] = t[i]->numel() > 0 ? t[i]->mutable_data_ptr() : nullptr;
  }
  *rows = t[1]->dim() == 3 ? t[1]->size(0) : -1;
  *n_obs = n_tensors == 5 && t[4]->dim() == 3 ? t[4]->size(0) : 0;
  if (*rows < 0 || *rows > INT32_MAX || *n_obs > INT32_MAX || !rows_of(*t[1], kv_row, *rows) || !rows_of(*t[2], kv_row, *rows)) return false;
  for (const int i : {0, 3}) {
    if (step ? t[i]->dim() != 2 || t[i]->size(0) != q_row[0] || t[i]->size(1) != q_row[1] : !rows_of(*t[i], q_row, *rows)) return false;
  }
  return n_tensors < 5 || rows_of(*t[4], q_row, *n_obs);
}

// `tensors`: (q, k_tail, v_tail, out) of a step, token_begin None; or (q, k, v, out[, q_obs]) of a block
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 9) {
    PyErr_SetString(PyExc_TypeError, "call takes nine arguments");
    return nullptr;
  }
  void *entry, *handle, *stream;
  int32_t layer, device, token_begin = 0;
  int64_t q_row[2], kv_row[2];
  PyObject* const list = args[3];
  const bool step = args[8] == Py_None;
  if (!address(args[0], &entry) || !entry || !address(args[1], &handle) || !handle || !small_int(args[2], &layer) || !PyTuple_CheckExact(list) ||
      !pair(args[4], q_row) || !pair(args[5], kv_row) || !small_int(args[6], &device) || !address(args[7], &stream) ||
      (!step && !small_int(args[8], &token_begin)))
    Py_RETURN_NONE;
  const Py_ssize_t n_tensors = PyTuple_GET_SIZE(list);
  if (n_tensors < 4 || n_tensors > (step ? 4 : kMostTensors)) Py_RETURN_NONE;
  void* p[kMostTensors];
  int64_t rows = -1, n_obs = 0;
  try {
    if (!plain_tensors(list, n_tensors, step, q_row, kv_row, device, p, &rows, &n_obs)) Py_RETURN_NONE;
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  int code;
  Py_BEGIN_ALLOW_THREADS;                    // (as ctypes does: a launch may have to wait)
  if (step)
    code = ((int (*)(void*, int32_t, const void*, const void*, const void*, int32_t, void*, void*))entry)(handle, layer, p[0], p[1], p[2],
                                                                                                     (int32_t)rows, p[3], stream);
  else if (n_tensors == 4)
    code = ((int (*)(void*, int32_t, int32_t, int32_t, const void*, const void*, const void*, void*, void*))entry)(
        handle, layer, token_begin, (int32_t)rows, p[0], p[1], p[2], p[3], stream);
  else
    code = ((int (*)(void*, int32_t, int32_t, int32_t, const void*, const void*, const void*, void*, const void*, int32_t, void*))entry)(
        handle, layer, token_begin, (int32_t)rows, p[0], p[1], p[2], p[3], p[4], (int32_t)n_obs, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

// ---- the calls of many sequences
struct Numbers {                  // bf16 rows [tokens, heads, d]
  void* at;
  int64_t token, head;
};
// (An address may have to be made, and torch may throw for it: like all that looks at tensors these belong where exceptions are caught.)
void* numbers_at(const at::Tensor* t) { return t->numel() > 0 ? t->mutable_data_ptr() : nullptr; }
bool numbers(PyObject* o, int64_t device, int64_t tokens, int64_t heads, int64_t d, Numbers* out) {
  const at::Tensor* t;
  if (!plain_of(o, device, at::kBFloat16, &t) || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != d || t->stride(2) != 1) return false;
  *out = Numbers{numbers_at(t), tokens > 1 ? t->stride(0) : 0, heads > 1 ? t->stride(1) : 0};
  return true;
}
// contiguous int32 numbers
bool whole(PyObject* o, int64_t device, const at::Tensor** out) { return plain_of(o, device, at::kInt, out) && (*out)->is_contiguous(); }
const int32_t* ints(const at::Tensor* t) { return t->numel() > 0 ? static_cast<const int32_t*>(t->const_data_ptr()) : nullptr; }

// The kvp_pages, by its address or by (address, k, v, k_exp, v_exp): tensors, or None without exponents, whose memory has to be what it says.
bool pages_of(PyObject* o, void** out) {
  if (!PyTuple_CheckExact(o)) return address(o, out) && *out;
  if (PyTuple_GET_SIZE(o) != 5 || !address(PyTuple_GET_ITEM(o, 0), out) || !*out) return false;
  const kvp_pages& p = *static_cast<const kvp_pages*>(*out);
  const void* const said[4] = {p.k, p.v, p.k_exp, p.v_exp};
  for (int i = 0; i < 4; ++i) {
    PyObject* const t = PyTuple_GET_ITEM(o, i + 1);
    if (t == Py_None ? said[i] != nullptr : !THPVariable_Check(t) || THPVariable_Unpack(t).const_data_ptr() != said[i]) return false;
  }
  return true;
}

// page_rows(entry, pages, n_kv_heads, head_dim, device, stream, k, v, seq_begin, table, first)
PyObject* page_rows(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 11) {
    PyErr_SetString(PyExc_TypeError, "page_rows takes eleven arguments");
    return nullptr;
  }
  void *entry, *pages, *stream;
  int32_t heads, d, device;
  if (!address(args[0], &entry) || !entry || !small_int(args[2], &heads) || !small_int(args[3], &d) || !small_int(args[4], &device) ||
      !address(args[5], &stream))
    Py_RETURN_NONE;
  kvp_rows rows;
  const int32_t *begin_at, *table_at, *first_at = nullptr;
  int32_t n_seqs, width;
  try {
    if (!pages_of(args[1], &pages)) Py_RETURN_NONE;
    const at::Tensor *k, *begin, *table, *first = nullptr;
    Numbers kn, vn;
    if (!plain_of(args[6], device, at::kBFloat16, &k) || k->dim() != 3 || k->size(0) > INT32_MAX) Py_RETURN_NONE;
    const int64_t n = k->size(0);
    if (!numbers(args[6], device, n, heads, d, &kn) || !numbers(args[7], device, n, heads, d, &vn)) Py_RETURN_NONE;
    if (!whole(args[8], device, &begin) || !whole(args[9], device, &table) || begin->dim() != 1 || table->dim() != 2) Py_RETURN_NONE;
    if (begin->size(0) > INT32_MAX || table->size(0) != begin->size(0) - 1 || table->size(1) > INT32_MAX) Py_RETURN_NONE;
    if (args[10] != Py_None && (!whole(args[10], device, &first) || first->dim() != 1 || first->size(0) != table->size(0))) Py_RETURN_NONE;
    rows = kvp_rows{kn.at, vn.at, kn.token, kn.head, vn.token, vn.head, (int32_t)n};
    n_seqs = (int32_t)table->size(0);
    width = (int32_t)table->size(1);
    begin_at = ints(begin);
    table_at = ints(table);
    if (first) first_at = ints(first);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  int code;
  Py_BEGIN_ALLOW_THREADS;
  code = ((decltype(&kvp_page_write))entry)((const kvp_pages*)pages, &rows, begin_at, table_at, width, first_at, n_seqs, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

// paged_decode(entry, pages, n_q_heads, head_dim, device, stream, q, table, lengths, out, workspace or its bytes, softmax_scale).  With a number of
// bytes the workspace is allocated here, for the stream that torch works on.
PyObject* paged_decode(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "paged_decode takes twelve arguments");
    return nullptr;
  }
  void *entry, *pages, *stream;
  int32_t heads, d, device, bytes = 0;
  if (!address(args[0], &entry) || !entry || !small_int(args[2], &heads) || !small_int(args[3], &d) || !small_int(args[4], &device) ||
      !address(args[5], &stream) || !PyFloat_CheckExact(args[11]))
    Py_RETURN_NONE;
  const bool own = small_int(args[10], &bytes);
  const int32_t *table_at, *lengths_at;
  void *out_at, *room_at;
  size_t room_bytes;
  at::Tensor made;
  Numbers q;
  int32_t n_seqs, width;
  try {
    if (!pages_of(args[1], &pages)) Py_RETURN_NONE;
    const at::Tensor *table, *lengths, *out, *room;
    if (!whole(args[7], device, &table) || !whole(args[8], device, &lengths) || table->dim() != 2 || lengths->dim() != 1) Py_RETURN_NONE;
    if (lengths->size(0) > INT32_MAX || table->size(0) != lengths->size(0) || table->size(1) > INT32_MAX) Py_RETURN_NONE;
    n_seqs = (int32_t)lengths->size(0);
    width = (int32_t)table->size(1);
    if (!numbers(args[6], device, n_seqs, heads, d, &q) || !plain(args[9], device, &out)) Py_RETURN_NONE;
    if (out->dim() != 3 || out->size(0) != n_seqs || out->size(1) != heads || out->size(2) != d) Py_RETURN_NONE;
    if (own) {
      made = at::empty({bytes}, at::TensorOptions().dtype(at::kByte).device(c10::Device(KVP_TENSOR_DEVICE, (c10::DeviceIndex)device)));
      room = &made;
    } else if (!plain_of(args[10], device, at::kByte, &room) || !room->is_contiguous()) {
      Py_RETURN_NONE;
    }
    table_at = ints(table);
    lengths_at = ints(lengths);
    out_at = numbers_at(out);
    room_at = numbers_at(room);
    room_bytes = (size_t)room->numel();
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  int code;
  const float scale = (float)PyFloat_AS_DOUBLE(args[11]);
  Py_BEGIN_ALLOW_THREADS;
  code = ((decltype(&kvp_paged_decode))entry)((const kvp_pages*)pages, q.at, q.token, q.head, heads, table_at, width, lengths_at, n_seqs, scale, out_at, room_at,
                                              room_bytes, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

// prompt(entry, device, stream, q, k, v, seq_begin, out, softmax_scale)
PyObject* prompt(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 9) {
    PyErr_SetString(PyExc_TypeError, "prompt takes nine arguments");
    return nullptr;
  }
  void *entry, *stream;
  int32_t device;
  if (!address(args[0], &entry) || !entry || !small_int(args[1], &device) || !address(args[2], &stream) || !PyFloat_CheckExact(args[8])) Py_RETURN_NONE;
  kvp_prompts p;
  try {
    const at::Tensor *qt, *kt, *begin;
    Numbers q, k, v, out;
    if (!plain_of(args[3], device, at::kBFloat16, &qt) || !plain_of(args[4], device, at::kBFloat16, &kt) || qt->dim() != 3 || kt->dim() != 3) Py_RETURN_NONE;
    const int64_t n = qt->size(0), hq = qt->size(1), d = qt->size(2), hkv = kt->size(1);
    if (n > INT32_MAX || hq > INT32_MAX || hkv > INT32_MAX || d > INT32_MAX) Py_RETURN_NONE;
    if (!numbers(args[3], device, n, hq, d, &q) || !numbers(args[4], device, n, hkv, d, &k) || !numbers(args[5], device, n, hkv, d, &v) ||
        !numbers(args[7], device, n, hq, d, &out))
      Py_RETURN_NONE;
    if (!whole(args[6], device, &begin) || begin->dim() != 1 || begin->size(0) < 1 || begin->size(0) > INT32_MAX) Py_RETURN_NONE;
    p = kvp_prompts{q.at, k.at, v.at, out.at, ints(begin), q.token, q.head, k.token, k.head, v.token, v.head, out.token, out.head,
                    (int32_t)n, (int32_t)(begin->size(0) - 1), (int32_t)hq, (int32_t)hkv, (int32_t)d, (float)PyFloat_AS_DOUBLE(args[8])};
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  int code;
  Py_BEGIN_ALLOW_THREADS;
  code = ((decltype(&kvp_prompt_attention))entry)(&p, stream);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(code);
}

#define KVP_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KVP_METHOD(call), KVP_METHOD(page_rows), KVP_METHOD(paged_decode), KVP_METHOD(prompt), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: that of the headers the module was built with, whose layouts of a tensor are part of its code
PyMODINIT_FUNC PyInit__fast_calls() {
  PyObject* const m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", KVP_TORCH_VERSION) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
