// Python binding of the calls that sit in a model's loop (laq_evict, laq_decode_attention, laq_qcache_store, and those of the
// 4-bit cache) as a CPython extension: the marshalling of binding.py and fp4.py in C++.
//
// A small call is bound by the host: the kernels of one layer's step take a few microseconds, and what
// Python spends on unpacking tensors, filling ctypes structures and making output tensors took 10 us per
// decode call and 20 us per eviction; here it is 2 to 4.
//
// Every function takes exactly what its namesake in binding.py or fp4.py takes (positionally, defaults filled in
// there) and returns None for anything out of the ordinary -- a tensor of another type, device or layout,
// an argument that is not a plain number, anything that throws (no memory for an output, a tensor without an
// address) -- without having launched anything: binding.py then walks its own checks and raises what it always
// raised, of the type it always had.  An error of the library comes back as its (negative) code.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string.h>

#include <vector>

#include "laq.h"
#include "laq_fp4.h"

namespace {

decltype(&laq_evict) fn_evict;
decltype(&laq_workspace_bytes) fn_workspace_bytes;
decltype(&laq_decode_attention) fn_decode_attention;
decltype(&laq_decode_workspace_bytes) fn_decode_workspace_bytes;
decltype(&laq_qcache_store) fn_qcache_store;
decltype(&laq_block_map) fn_block_map;
decltype(&laq_fp4_store) fn_fp4_store;
decltype(&laq_fp4_compact) fn_fp4_compact;
decltype(&laq_fp4_load) fn_fp4_load;
decltype(&laq_fp4_attention) fn_fp4_attention;
decltype(&laq_fp4_attention_workspace_bytes) fn_fp4_attention_workspace_bytes;
PyObject* get_device;      // torch._C._cuda_getDevice
PyObject* get_stream;      // torch._C._cuda_getCurrentRawStream

bool is_none(PyObject* o) { return o == Py_None; }
bool is_text(PyObject* o, const char* text) { return PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, text) == 0; }

// tensor on a GPU, or null
const at::Tensor* gpu_tensor(PyObject* o) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return LAQ_BF16;
  if (t.scalar_type() == at::kFloat) return LAQ_F32;
  return -1;
}

bool aligned(const at::Tensor& t, uintptr_t to = 16) { return reinterpret_cast<uintptr_t>(t.data_ptr()) % to == 0; }

// a caller-supplied output: dense, of the type and on the device, large enough, aligned
const at::Tensor* output(PyObject* o, at::ScalarType type, int64_t numel, const at::Tensor& like) {
  const at::Tensor* t = gpu_tensor(o);
  if (!t || t->device() != like.device() || t->scalar_type() != type || !t->is_contiguous() || t->numel() < numel || !aligned(*t))
    return nullptr;
  return t;
}

bool as_int(PyObject* o, long long* v) {
  if (!PyLong_CheckExact(o)) return false;
  *v = PyLong_AsLongLong(o);
  if (*v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return *v >= INT32_MIN && *v <= INT32_MAX;
}

// list or tuple of whole numbers
bool as_ints(PyObject* o, std::vector<int32_t>* out) {
  if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
  PyObject** items = PySequence_Fast_ITEMS(o);
  out->resize(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    long long v;
    if (!as_int(items[i], &v)) return false;
    (*out)[i] = (int32_t)v;
  }
  return true;
}

// stream of the calling thread on the current device
bool current_stream(void** out) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  PyObject* st = dev ? PyObject_CallOneArg(get_stream, dev) : nullptr;
  Py_XDECREF(dev);
  if (!st) return false;
  *out = PyLong_AsVoidPtr(st);
  Py_DECREF(st);
  return !PyErr_Occurred();
}

at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}

PyObject* none() { Py_RETURN_NONE; }
// after a C++ exception: one that carries a Python exception (a dispatch mode raised it) leaves that set
PyObject* thrown() { return PyErr_Occurred() ? nullptr : none(); }

// rows of the packed outputs; false: a budget the library will refuse
bool packed_rows(const std::vector<int32_t>& budget, int64_t Hkv, int64_t L, int64_t* rows) {
  int64_t total = 0;
  for (const int32_t b : budget) {
    if (b < 1) return false;
    total += Hkv * (b < L ? b : L);
  }
  *rows = total;
  return true;
}

// evict(q_win, k, v, budget, pool_kernel, scale, scores, idx, k_out, v_out, ws, q_pos, keep, pool_mode,
//       want_scores, block_table, L, choose) -> (scores, idx, k_out, v_out) | error code | None
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 18) return none();
    const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = is_none(a[2]) ? nullptr : gpu_tensor(a[2]);
    if (!q || !k || (!v && !is_none(a[2])) || q->dim() != 4 || k->dim() != 4 || !q->is_contiguous() || k->stride(3) != 1) return none();
    const int dt = dtype_code(*k);
    if (dt < 0 || q->scalar_type() != k->scalar_type() || q->device() != k->device() || !aligned(*q) || !aligned(*k)) return none();
    laq_shape sh;
    memset(&sh, 0, sizeof sh);
    const int64_t n = q->size(0), Hkv = k->size(1), d = q->size(3);
    int64_t L = k->size(2);
    if (k->size(3) != d) return none();
    if (is_none(a[15])) {
      long long want_L;
      if (!is_none(a[16]) && (!as_int(a[16], &want_L) || want_L != L)) return none();
      if (k->size(0) != n) return none();
      if (!k->is_contiguous()) {
        sh.kv_stride_inst = k->stride(0);
        sh.kv_stride_head = k->stride(1);
        sh.kv_stride_row = k->stride(2);
      }
    } else {
      const at::Tensor* table = gpu_tensor(a[15]);
      long long want_L;
      if (!table || !as_int(a[16], &want_L) || want_L < 1) return none();
      const int64_t rows = k->size(2);
      L = want_L;
      if (table->device() != k->device() || table->scalar_type() != at::kInt || table->dim() != 2 || !table->is_contiguous() ||
          rows < 1 || rows % 256 || rows > INT32_MAX || table->size(0) != n || table->size(1) != (L + rows - 1) / rows)
        return none();
      if (k->stride(1) != rows * d || k->stride(2) != d) {
        sh.kv_stride_head = k->stride(1);
        sh.kv_stride_row = k->stride(2);
      }
      sh.block_table = table->data_ptr<int32_t>();
      sh.block_rows = (int32_t)rows;
      sh.kv_stride_block = k->stride(0);
    }
    if (n < 1 || n > INT32_MAX || q->size(1) > INT32_MAX || Hkv > INT32_MAX || L > INT32_MAX || q->size(2) > INT32_MAX) return none();
    std::vector<int32_t> budget, pos;
    int64_t rows = 0;
    long long pool, keep = -1;
    if (!as_ints(a[3], &budget) || (int64_t)budget.size() != n || !packed_rows(budget, Hkv, L, &rows) || !as_int(a[4], &pool)) return none();
    const double scale = PyFloat_CheckExact(a[5]) ? PyFloat_AS_DOUBLE(a[5]) : -1.0;
    if (!PyFloat_CheckExact(a[5])) return none();
    if (!is_none(a[11])) {
      if (!as_ints(a[11], &pos) || (int64_t)pos.size() != q->size(2)) return none();
      sh.q_pos = pos.data();
    }
    if (!is_none(a[12]) && !as_int(a[12], &keep)) return none();
    if (is_text(a[13], "max")) sh.pool_mode = LAQ_POOL_MAX;
    else if (is_text(a[13], "avg")) sh.pool_mode = LAQ_POOL_AVG;
    else return none();
    if (is_text(a[17], "auto")) sh.score_choice = LAQ_CHOOSE_AUTO;
    else if (is_text(a[17], "two-pass")) sh.score_choice = LAQ_CHOOSE_TWO_PASS;
    else if (is_text(a[17], "single-read")) sh.score_choice = LAQ_CHOOSE_SINGLE_READ;
    else return none();
    if (!PyBool_Check(a[14])) return none();
    if (v) {
      if (v->scalar_type() != k->scalar_type() || v->device() != k->device() || v->sizes() != k->sizes() ||
          v->strides() != k->strides() || !aligned(*v))
        return none();
    } else if (!is_none(a[9])) {
      return none();
    }
    sh.n_inst = (int32_t)n; sh.Hq = (int32_t)q->size(1); sh.Hkv = (int32_t)Hkv; sh.d = (int32_t)d; sh.L = (int32_t)L;
    sh.W = (int32_t)q->size(2); sh.dtype = dt; sh.scale = (float)scale; sh.keep = (int32_t)keep;

    // outputs: what the caller gave, else new ones
    at::Tensor made[5];
    const at::Tensor* out[5] = {};         // scores, idx, k_out, v_out, ws
    const at::ScalarType type[4] = {at::kFloat, at::kInt, k->scalar_type(), k->scalar_type()};
    const int64_t numel[4] = {n * Hkv * L, rows, rows * d, rows * d};
    for (int i = 0; i < 4; ++i)
      if (!is_none(a[6 + i]) && !(out[i] = output(a[6 + i], type[i], numel[i], *k))) return none();
    const size_t need = fn_workspace_bytes(&sh);
    if (need == 0) return none();
    if (!is_none(a[10])) {
      out[4] = gpu_tensor(a[10]);
      if (!out[4] || out[4]->device() != k->device() || !out[4]->is_contiguous() || !aligned(*out[4], 256)) return none();
    }
    if (!out[0] && a[14] == Py_True) out[0] = &(made[0] = make({n, Hkv, L}, at::kFloat, *k));
    if (!out[1]) out[1] = &(made[1] = make({rows}, at::kInt, *k));
    if (!out[2]) out[2] = &(made[2] = make({rows, d}, type[2], *k));
    if (v && !out[3]) out[3] = &(made[3] = make({rows, d}, type[3], *k));
    if (!out[4]) out[4] = &(made[4] = make({(int64_t)need}, at::kByte, *k));
    void* stream;
    if (!current_stream(&stream)) return nullptr;
    // (a tensor without memory throws when it is asked for its address: not where the GIL is released)
    int rc;
    const size_t ws_bytes = out[4]->numel() * out[4]->element_size();
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v ? v->data_ptr() : nullptr;
    void* op[5];
    for (int i = 0; i < 5; ++i) op[i] = out[i] ? out[i]->data_ptr() : nullptr;
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_evict(&sh, qp, kp, vp, budget.data(), (int)pool, static_cast<float*>(op[0]), static_cast<int32_t*>(op[1]), op[2],
                  op[3], op[4], ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    PyObject* res = PyTuple_New(4);
    if (!res) return nullptr;
    for (int i = 0; i < 4; ++i) {
      PyObject* o;
      if (!is_none(a[6 + i]) || !out[i]) {           // the caller's own, or no such output
        o = a[6 + i];
        Py_INCREF(o);
      } else {
        o = THPVariable_Wrap(std::move(made[i]));
        if (!o) {
          Py_DECREF(res);
          return nullptr;
        }
      }
      PyTuple_SET_ITEM(res, i, o);
    }
    return res;
  } catch (const std::exception&) {
    return thrown();
  }
}

// decode(q, k_c, v_c, budget, Hkv, L, scale, out, ws, split) -> out | error code | None
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 10) return none();
    const at::Tensor *q = gpu_tensor(a[0]), *k = gpu_tensor(a[1]), *v = gpu_tensor(a[2]);
    if (!q || !k || !v || q->dim() != 3 || k->dim() != 2 || v->dim() != 2) return none();
    const int dt = dtype_code(*q);
    std::vector<int32_t> budget;
    long long Hkv, L;
    int64_t rows = 0;
    const int64_t n = q->size(0), Hq = q->size(1), d = q->size(2);
    if (dt < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() || k->device() != q->device() ||
        v->device() != q->device() || !q->is_contiguous() || !k->is_contiguous() || !v->is_contiguous() || !as_ints(a[3], &budget) ||
        (int64_t)budget.size() != n || !as_int(a[4], &Hkv) || !as_int(a[5], &L) || Hkv < 1 || L < 1 || !packed_rows(budget, Hkv, L, &rows) ||
        k->size(0) != rows || k->size(1) != d || v->size(0) != rows || v->size(1) != d || !PyFloat_CheckExact(a[6]) || !PyBool_Check(a[9]) ||
        n < 1 || n > INT32_MAX || Hq > INT32_MAX)
      return none();
    laq_shape sh;
    memset(&sh, 0, sizeof sh);
    sh.n_inst = (int32_t)n; sh.Hq = (int32_t)Hq; sh.Hkv = (int32_t)Hkv; sh.d = (int32_t)d; sh.L = (int32_t)L; sh.W = 1; sh.dtype = dt;
    sh.scale = (float)PyFloat_AS_DOUBLE(a[6]);
    at::Tensor made, scratch;
    const at::Tensor *out = nullptr, *ws = nullptr;
    if (!is_none(a[7]) && !(out = output(a[7], at::kFloat, n * Hq * d, *q))) return none();
    if (a[9] == Py_True) {
      if (!is_none(a[8])) {
        if (!(ws = gpu_tensor(a[8]))) return none();
      } else if (const size_t need = fn_decode_workspace_bytes(&sh, budget.data())) {
        ws = &(scratch = make({(int64_t)need}, at::kByte, *q));
      }
    }
    if (!out) out = &(made = make({n, Hq, d}, at::kFloat, *q));
    void* stream;
    if (!current_stream(&stream)) return nullptr;
    int rc;
    const size_t ws_bytes = ws ? ws->numel() * ws->element_size() : 0;
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    void *op = out->data_ptr(), *wp = ws ? ws->data_ptr() : nullptr;
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_decode_attention(&sh, qp, kp, vp, budget.data(), static_cast<float*>(op), wp, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    if (!is_none(a[7])) {
      Py_INCREF(a[7]);
      return a[7];
    }
    return THPVariable_Wrap(std::move(made));
  } catch (const std::exception&) {
    return thrown();
  }
}

// qcache_store(q_cache, q_step, t) -> q_cache | error code | None
PyObject* qcache_store(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 3) return none();
    const at::Tensor *c = gpu_tensor(a[0]), *q = gpu_tensor(a[1]);
    long long t;
    if (!c || !q || c->dim() != 4 || q->dim() != 3 || !c->is_contiguous() || !q->is_contiguous() || c->scalar_type() != q->scalar_type() ||
        c->device() != q->device() || q->size(0) != c->size(0) || q->size(1) != c->size(1) || q->size(2) != c->size(3) || !as_int(a[2], &t))
      return none();
    const int dt = dtype_code(*c);
    if (dt < 0 || c->size(0) < 1 || c->size(0) > INT32_MAX || c->size(1) > INT32_MAX || c->size(2) < 1 || c->size(2) > INT32_MAX) return none();
    laq_shape sh;
    memset(&sh, 0, sizeof sh);
    sh.n_inst = (int32_t)c->size(0); sh.Hq = sh.Hkv = (int32_t)c->size(1); sh.d = (int32_t)c->size(3);
    sh.L = sh.W = (int32_t)c->size(2); sh.dtype = dt;
    void* stream;
    if (!current_stream(&stream)) return nullptr;
    int rc;
    const void* qp = q->data_ptr();
    void* cp = c->data_ptr();
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_qcache_store(&sh, qp, (int32_t)t, cp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    Py_INCREF(a[0]);
    return a[0];
  } catch (const std::exception&) {
    return thrown();
  }
}

// ---- the 4-bit cache -----------------------------------------------------------------------

// stream of the calling thread, if `device` is the current one; else false, with or without a Python exception
bool stream_on(const at::Device& device, void** out) {
  PyObject* dev = PyObject_CallNoArgs(get_device);
  if (!dev) return false;
  const long current = PyLong_AsLong(dev);
  PyObject* st = current == device.index() ? PyObject_CallOneArg(get_stream, dev) : nullptr;
  Py_DECREF(dev);
  if (!st) return false;
  *out = PyLong_AsVoidPtr(st);
  Py_DECREF(st);
  return !PyErr_Occurred();
}

// dense int32 tensor of at least `numel` entries on the device
const at::Tensor* ints(PyObject* o, const at::Device& device, int64_t numel) {
  const at::Tensor* t = gpu_tensor(o);
  return t && t->device() == device && t->scalar_type() == at::kInt && t->is_contiguous() && t->numel() >= numel ? t : nullptr;
}

// an Fp4Cache: its four tensors, and what the library takes
bool fp4_cache(PyObject* o, laq_fp4_cache* c, const at::Tensor** first) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i) {
    t[i] = gpu_tensor(PyTuple_GET_ITEM(o, i));
    if (!t[i] || t[i]->dim() != 4 || t[i]->scalar_type() != at::kByte || t[i]->device() != t[0]->device() || t[i]->stride(3) != 1) return false;
  }
  for (int i = 1; i < 4; ++i)
    for (int x = 0; x < 3; ++x)
      if (t[i]->size(x) != t[0]->size(x) || t[0]->size(x) > INT32_MAX) return false;
  if (t[0]->size(3) > 128 || t[0]->size(3) != t[2]->size(3) || t[1]->size(3) * 16 != t[0]->size(3) || t[3]->size(3) != t[1]->size(3) ||
      t[2]->strides() != t[0]->strides() || t[3]->strides() != t[1]->strides())
    return false;
  memset(c, 0, sizeof *c);
  c->k = static_cast<uint8_t*>(t[0]->data_ptr());
  c->k_scale = static_cast<uint8_t*>(t[1]->data_ptr());
  c->v = static_cast<uint8_t*>(t[2]->data_ptr());
  c->v_scale = static_cast<uint8_t*>(t[3]->data_ptr());
  c->n_blocks = (int32_t)t[0]->size(0);
  c->Hkv = (int32_t)t[0]->size(1);
  c->block_rows = (int32_t)t[0]->size(2);
  c->d = (int32_t)(2 * t[0]->size(3));
  if (c->block_rows < 1) return false;
  if (!t[0]->is_contiguous() || !t[1]->is_contiguous()) {
    c->stride_block = t[0]->stride(0);
    c->stride_head = t[0]->stride(1);
    c->stride_row = t[0]->stride(2);
    c->scale_stride_block = t[1]->stride(0);
    c->scale_stride_head = t[1]->stride(1);
    c->scale_stride_row = t[1]->stride(2);
  }
  *first = t[0];
  return true;
}

// [tokens, heads, d] with contiguous rows on the device, its strides as the library takes them
bool token_rows(const at::Tensor* t, const at::Device& device, int64_t d, int64_t* token, int64_t* head) {
  if (!t || t->device() != device || t->dim() != 3 || t->size(2) != d || t->stride(2) != 1 || !aligned(*t) || dtype_code(*t) < 0) return false;
  *token = *head = 0;
  if (!t->is_contiguous()) {
    *token = t->stride(0);
    *head = t->stride(1);
  }
  return true;
}

PyObject* own_or_made(PyObject* given, at::Tensor* made) {
  if (!is_none(given) || !made->defined()) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(std::move(*made));
}

PyObject* pair(PyObject* a, PyObject* b) {
  if (!a || !b) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    return nullptr;
  }
  PyObject* res = PyTuple_Pack(2, a, b);
  Py_DECREF(a);
  Py_DECREF(b);
  return res;
}

// block_map(add, rows, block_table, free_blocks, state, block_rows, start, slots, n_slots) -> (start, slots) | error code | None
PyObject* block_map(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 9) return none();
    const at::Tensor* rows = gpu_tensor(a[1]);
    if (!rows) return none();
    const int64_t n = rows->numel();
    const at::Device dev = rows->device();
    const at::Tensor *add = ints(a[0], dev, n), *table = ints(a[2], dev, n), *list = ints(a[3], dev, 1), *state = ints(a[4], dev, 4);
    long long block_rows, n_slots = 0;
    if (!ints(a[1], dev, n) || !add || !table || !list || !state || add->numel() != n || table->dim() != 2 || table->size(0) != n || n > INT32_MAX ||
        table->size(1) > INT32_MAX || list->numel() > INT32_MAX || !as_int(a[5], &block_rows) || (!is_none(a[8]) && (!as_int(a[8], &n_slots) || n_slots < 0)))
      return none();
    const at::Tensor *start = nullptr, *slots = nullptr;
    if (!is_none(a[6]) && !(start = ints(a[6], dev, n + 1))) return none();
    if (!is_none(a[7]) && !(slots = ints(a[7], dev, n_slots))) return none();
    void* stream;
    if (!stream_on(dev, &stream)) return PyErr_Occurred() ? nullptr : none();
    at::Tensor made[2];
    if (!is_none(a[8])) {
      if (!start) start = &(made[0] = make({n + 1}, at::kInt, *rows));
      if (!slots) slots = &(made[1] = make({(int64_t)n_slots}, at::kInt, *rows));
    }
    int rc;
    const int32_t* add_p = add->data_ptr<int32_t>();
    int32_t *rows_p = rows->data_ptr<int32_t>(), *table_p = table->data_ptr<int32_t>(), *list_p = list->data_ptr<int32_t>(), *state_p = state->data_ptr<int32_t>();
    int32_t *start_p = start ? start->data_ptr<int32_t>() : nullptr, *slots_p = slots ? slots->data_ptr<int32_t>() : nullptr;
    const int64_t count = slots ? slots->numel() : 0;
    const int32_t n_blocks = (int32_t)list->numel(), width = (int32_t)table->size(1);
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_block_map((int32_t)n, (int32_t)block_rows, n_blocks, width, add_p, rows_p, table_p, list_p, state_p, start_p, slots_p, count, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    return pair(own_or_made(a[6], &made[0]), own_or_made(a[7], &made[1]));
  } catch (const std::exception&) {
    return thrown();
  }
}

// fp4_store(cache, k, v, slots) -> True | error code | None
PyObject* fp4_store(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 4) return none();
    laq_fp4_cache c;
    const at::Tensor *first, *k = is_none(a[1]) ? nullptr : gpu_tensor(a[1]), *v = is_none(a[2]) ? nullptr : gpu_tensor(a[2]);
    if (!fp4_cache(a[0], &c, &first) || (!k && !is_none(a[1])) || (!v && !is_none(a[2])) || (!k && !v)) return none();
    const at::Device dev = first->device();
    const at::Tensor& like = k ? *k : *v;
    int64_t token, head, v_token, v_head;
    if (!token_rows(&like, dev, c.d, &token, &head) || like.size(1) != c.Hkv) return none();
    if (k && v && (!token_rows(v, dev, c.d, &v_token, &v_head) || v->sizes() != k->sizes() || v->scalar_type() != k->scalar_type() || v_token != token || v_head != head))
      return none();
    const at::Tensor* slots = ints(a[3], dev, like.size(0));
    if (!slots) return none();
    void* stream;
    if (!stream_on(dev, &stream)) return PyErr_Occurred() ? nullptr : none();
    int rc;
    const int dt = dtype_code(like);
    const int64_t n_tokens = like.size(0);
    const void *kp = k ? k->data_ptr() : nullptr, *vp = v ? v->data_ptr() : nullptr;
    const int32_t* sp = slots->data_ptr<int32_t>();
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_fp4_store(&c, dt, n_tokens, kp, vp, token, head, sp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
  } catch (const std::exception&) {
    return thrown();
  }
}

// fp4_compact(cache, k, v, idx, budget, slots) -> True | error code | None (paged sources: fp4.py)
PyObject* fp4_compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 6) return none();
    laq_fp4_cache c;
    const at::Tensor *first, *k = gpu_tensor(a[1]), *v = is_none(a[2]) ? nullptr : gpu_tensor(a[2]);
    if (!fp4_cache(a[0], &c, &first) || !k || (!v && !is_none(a[2])) || k->dim() != 4 || k->stride(3) != 1) return none();
    const at::Device dev = first->device();
    const int dt = dtype_code(*k);
    std::vector<int32_t> budget;
    int64_t rows = 0;
    const int64_t n = k->size(0), L = k->size(2);
    if (dt < 0 || k->device() != dev || k->size(1) != c.Hkv || k->size(3) != c.d || !aligned(*k) || n < 1 || n > INT32_MAX || L > INT32_MAX ||
        !as_ints(a[4], &budget) || (int64_t)budget.size() != n || !packed_rows(budget, 1, L, &rows))
      return none();
    if (v && (v->scalar_type() != k->scalar_type() || v->device() != dev || v->sizes() != k->sizes() || v->strides() != k->strides() || !aligned(*v))) return none();
    const at::Tensor *idx = ints(a[3], dev, rows * c.Hkv), *slots = ints(a[5], dev, rows);
    if (!idx || !slots) return none();
    laq_shape sh;
    memset(&sh, 0, sizeof sh);
    sh.n_inst = (int32_t)n; sh.Hq = sh.Hkv = c.Hkv; sh.d = c.d; sh.L = (int32_t)L; sh.W = 1; sh.dtype = dt;
    if (!k->is_contiguous()) {
      sh.kv_stride_inst = k->stride(0);
      sh.kv_stride_head = k->stride(1);
      sh.kv_stride_row = k->stride(2);
    }
    void* stream;
    if (!stream_on(dev, &stream)) return PyErr_Occurred() ? nullptr : none();
    int rc;
    const void *kp = k->data_ptr(), *vp = v ? v->data_ptr() : nullptr;
    const int32_t *ip = idx->data_ptr<int32_t>(), *sp = slots->data_ptr<int32_t>();
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_fp4_compact(&sh, kp, vp, ip, budget.data(), &c, sp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
  } catch (const std::exception&) {
    return thrown();
  }
}

// fp4_load(cache, slots, dtype, k, v) -> (k, v) | error code | None
PyObject* fp4_load(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 5) return none();
    laq_fp4_cache c;
    const at::Tensor* first;
    if (!fp4_cache(a[0], &c, &first) || !THPDtype_Check(a[2])) return none();
    const at::Device dev = first->device();
    const at::ScalarType type = reinterpret_cast<THPDtype*>(a[2])->scalar_type;
    const at::Tensor* slots = ints(a[1], dev, 0);
    if (!slots || (type != at::kBFloat16 && type != at::kFloat)) return none();
    const int64_t n_tokens = slots->numel();
    const at::Tensor* out[2] = {};
    at::Tensor made[2];
    for (int i = 0; i < 2; ++i)
      if (!is_none(a[3 + i]) && !(out[i] = output(a[3 + i], type, n_tokens * c.Hkv * c.d, *first))) return none();
    void* stream;
    if (!stream_on(dev, &stream)) return PyErr_Occurred() ? nullptr : none();
    for (int i = 0; i < 2; ++i)
      if (!out[i]) out[i] = &(made[i] = make({n_tokens, c.Hkv, c.d}, type, *first));
    int rc;
    const int32_t* sp = slots->data_ptr<int32_t>();
    void *kp = out[0]->data_ptr(), *vp = out[1]->data_ptr();
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_fp4_load(&c, type == at::kFloat ? LAQ_F32 : LAQ_BF16, n_tokens, sp, kp, vp, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    return pair(own_or_made(a[3], &made[0]), own_or_made(a[4], &made[1]));
  } catch (const std::exception&) {
    return thrown();
  }
}

// fp4_attention(q, cache, block_table, rows, start, max_rows, scale, out, lse, want_lse, ws, split) -> out | (out, lse) | error code | None
PyObject* fp4_attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  try {
    if (n_args != 12) return none();
    laq_fp4_cache c;
    const at::Tensor *first, *q = gpu_tensor(a[0]);
    int64_t token, head;
    if (!fp4_cache(a[1], &c, &first)) return none();
    const at::Device dev = first->device();
    if (!token_rows(q, dev, c.d, &token, &head)) return none();
    const int64_t T = q->size(0), Hq = q->size(1);
    const at::Tensor* table = ints(a[2], dev, 0);
    if (!table || table->dim() != 2 || table->size(0) < 1 || table->size(0) > INT32_MAX || table->size(1) > INT32_MAX / c.block_rows || Hq > INT32_MAX) return none();
    const int64_t n = table->size(0), width = table->size(1);
    const at::Tensor *rows = ints(a[3], dev, n), *start = is_none(a[4]) ? nullptr : ints(a[4], dev, n + 1);
    long long most = width * c.block_rows;
    if (!rows || (!start && (!is_none(a[4]) || T != n)) || (!is_none(a[5]) && !as_int(a[5], &most)) || !PyFloat_CheckExact(a[6]) || !PyBool_Check(a[9]) ||
        !PyBool_Check(a[11]))
      return none();
    if (most < 1) most = 1;
    const int dt = dtype_code(*q);
    const at::Tensor *out = nullptr, *lse = nullptr, *ws = nullptr;
    at::Tensor made[2], scratch;
    if (!is_none(a[7]) && !(out = output(a[7], q->scalar_type(), T * Hq * c.d, *q))) return none();
    if (!is_none(a[8]) && !(lse = output(a[8], at::kFloat, T * Hq, *q))) return none();
    if (!is_none(a[10])) {
      ws = gpu_tensor(a[10]);
      if (!ws || ws->device() != dev || !ws->is_contiguous()) return none();
    }
    void* stream;
    if (!stream_on(dev, &stream)) return PyErr_Occurred() ? nullptr : none();
    if (a[11] == Py_False) {
      ws = nullptr;
    } else if (!ws) {
      if (const size_t need = fn_fp4_attention_workspace_bytes(&c, (int32_t)Hq, dt, (int32_t)n, T, (int32_t)most))
        ws = &(scratch = make({(int64_t)need}, at::kByte, *q));
    }
    if (!out) out = &(made[0] = make({T, Hq, c.d}, q->scalar_type(), *q));
    if (!lse && a[9] == Py_True) lse = &(made[1] = make({T, Hq}, at::kFloat, *q));
    int rc;
    const size_t ws_bytes = ws ? ws->numel() * ws->element_size() : 0;
    const void* qp = q->data_ptr();
    const int32_t *tp = table->data_ptr<int32_t>(), *rp = rows->data_ptr<int32_t>(), *stp = start ? start->data_ptr<int32_t>() : nullptr;
    void *op = out->data_ptr(), *wp = ws ? ws->data_ptr() : nullptr;
    float* lp = lse ? static_cast<float*>(lse->data_ptr()) : nullptr;
    const float scale = (float)PyFloat_AS_DOUBLE(a[6]);
    Py_BEGIN_ALLOW_THREADS;
    rc = fn_fp4_attention(&c, (int32_t)Hq, dt, scale, (int32_t)n, T, stp, qp, token, head, tp, (int32_t)width, rp, (int32_t)most, op, lp, wp, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != LAQ_OK) return PyLong_FromLong(rc);
    PyObject* o = own_or_made(a[7], &made[0]);
    return lse ? pair(o, own_or_made(a[8], &made[1])) : o;
  } catch (const std::exception&) {
    return thrown();
  }
}

// bind_fp4(addresses of laq_block_map, laq_fp4_store, laq_fp4_compact, laq_fp4_load, laq_fp4_attention, laq_fp4_attention_workspace_bytes)
PyObject* bind_fp4(PyObject*, PyObject* args) {
  unsigned long long f[6];
  if (!PyArg_ParseTuple(args, "KKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5])) return nullptr;
  fn_block_map = reinterpret_cast<decltype(fn_block_map)>(f[0]);
  fn_fp4_store = reinterpret_cast<decltype(fn_fp4_store)>(f[1]);
  fn_fp4_compact = reinterpret_cast<decltype(fn_fp4_compact)>(f[2]);
  fn_fp4_load = reinterpret_cast<decltype(fn_fp4_load)>(f[3]);
  fn_fp4_attention = reinterpret_cast<decltype(fn_fp4_attention)>(f[4]);
  fn_fp4_attention_workspace_bytes = reinterpret_cast<decltype(fn_fp4_attention_workspace_bytes)>(f[5]);
  Py_RETURN_NONE;
}

// bind(addresses of laq_evict, laq_workspace_bytes, laq_decode_attention, laq_decode_workspace_bytes, laq_qcache_store,
//      torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long f[5];
  PyObject *dev, *st;
  if (!PyArg_ParseTuple(args, "KKKKKOO", &f[0], &f[1], &f[2], &f[3], &f[4], &dev, &st)) return nullptr;
  fn_evict = reinterpret_cast<decltype(fn_evict)>(f[0]);
  fn_workspace_bytes = reinterpret_cast<decltype(fn_workspace_bytes)>(f[1]);
  fn_decode_attention = reinterpret_cast<decltype(fn_decode_attention)>(f[2]);
  fn_decode_workspace_bytes = reinterpret_cast<decltype(fn_decode_workspace_bytes)>(f[3]);
  fn_qcache_store = reinterpret_cast<decltype(fn_qcache_store)>(f[4]);
  Py_INCREF(dev);
  Py_INCREF(st);
  get_device = dev;
  get_stream = st;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(evict)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode)), METH_FASTCALL, nullptr},
    {"qcache_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qcache_store)), METH_FASTCALL, nullptr},
    {"bind_fp4", bind_fp4, METH_VARARGS, nullptr},
    {"block_map", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_map)), METH_FASTCALL, nullptr},
    {"fp4_store", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_store)), METH_FASTCALL, nullptr},
    {"fp4_compact", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_compact)), METH_FASTCALL, nullptr},
    {"fp4_load", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_load)), METH_FASTCALL, nullptr},
    {"fp4_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_attention)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
