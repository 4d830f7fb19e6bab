// The calls on a 4-bit cache taken straight from torch tensors (module _qc_torch, used by quant.py).
//
// What a call checks and packs is some forty tensor attributes.  An attention call, its allocations and its launch took the host
// 28 us from Python through ctypes, more than the kernel runs for a small batch; from here they take 8.  The calls keep nothing, enqueue on the current stream of the tensors' device, and raise ValueError for
// arguments that do not fit and QcError for a status of the library.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "../../include/qc.h"

namespace {

PyObject* g_qc_error = nullptr;

struct BadArgument : std::exception {
  std::string text;
  explicit BadArgument(std::string t) : text(std::move(t)) {}
  const char* what() const noexcept override { return text.c_str(); }
};
struct PythonError {};   // a Python exception is set

const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw BadArgument(std::string(name) + " has to be a tensor");
  return THPVariable_Unpack(o);
}

int64_t int_of(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  return v;
}
// an argument that the library takes as 32 bits: what does not fit there fits nowhere
int32_t int32_of(PyObject* o, const char* name) {
  const int64_t v = int_of(o);
  if (v < INT32_MIN || v > INT32_MAX) throw BadArgument(std::string(name) + " is out of range");
  return static_cast<int32_t>(v);
}
int32_t size32(int64_t v, const char* name) {
  if (v > INT32_MAX) throw BadArgument(std::string(name) + " is too large");
  return static_cast<int32_t>(v);
}

int32_t device_of(const at::Tensor& t, const char* name) {
  if (!t.is_cuda()) throw BadArgument(std::string(name) + " has to be on a CUDA device (there is no CPU fallback)");
  return t.get_device();
}

bool on(const at::Tensor& t, int32_t index) { return t.is_cuda() && t.get_device() == index; }
std::string cuda_name(int32_t index) { return "cuda:" + std::to_string(index); }

// Dense int32 tensor (null for None).  count < 0: any number of entries.
int32_t* ints(PyObject* o, const char* name, int32_t index, int64_t count = -1) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor_of(o, name);
  if (t.scalar_type() != at::kInt || !on(t, index) || !t.is_contiguous()) throw BadArgument(std::string(name) + " has to be a dense int32 tensor on " + cuda_name(index));
  if (count >= 0 && t.numel() != count)
    throw BadArgument(std::string(name) + " has " + std::to_string(t.numel()) + " entries, not " + std::to_string(count));
  return static_cast<int32_t*>(t.data_ptr());
}

void* pool_of(const at::Tensor& t, const char* name, int64_t row, int32_t index) {
  if (t.scalar_type() != at::kByte || !on(t, index) || !t.is_contiguous() || t.dim() != 2 || t.size(1) != row)
    throw BadArgument(std::string(name) + " has to be a dense uint8 tensor [pages, " + std::to_string(row) + "] on " + cuda_name(index) +
                      " (heads * page size * (head_dim / 2 + 4) bytes a page)");
  return t.data_ptr();
}

// Token stride of bf16 [tokens, heads, head_dim] rows whose heads are dense (0 for a single token).
int64_t rows_of(const at::Tensor& t, const char* name, int32_t index) {
  if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || !on(t, index))
    throw BadArgument(std::string(name) + " has to be a bfloat16 tensor [tokens, heads, head_dim] on " + cuda_name(index));
  if ((t.stride(2) != 1 && t.size(2) > 1) || (t.stride(1) != t.size(2) && t.size(1) > 1)) throw BadArgument(std::string(name) + ": the heads of a token have to be dense");
  return t.size(0) > 1 ? t.stride(0) : 0;
}

void check(int32_t status, const char* where) {
  if (status == QC_OK) return;
  PyObject* e = g_qc_error ? PyObject_CallFunction(g_qc_error, "is", status, where) : nullptr;
  if (e) {
    PyErr_SetObject(g_qc_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, where);
  }
  throw PythonError{};
}

void* stream_of(int32_t index) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(index)).stream(); }

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject* x = THPVariable_Wrap(a);
  PyObject* y = x ? THPVariable_Wrap(b) : nullptr;
  PyObject* t = y ? PyTuple_New(2) : nullptr;
  if (!t) {
    Py_XDECREF(x);
    Py_XDECREF(y);
    throw PythonError{};
  }
  PyTuple_SET_ITEM(t, 0, x);
  PyTuple_SET_ITEM(t, 1, y);
  return t;
}

void need_args(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) throw BadArgument("wrong number of arguments");
}

// No C++ exception leaves a call.
template <typename Fn>
PyObject* guarded(Fn fn) {
  try {
    return fn();
  } catch (const PythonError&) {
  } catch (const BadArgument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// ---- page tables: a table is (packed structure, device, rows) -----------------------------------------------

PyObject* py_table(PyObject*, PyObject* const* a, Py_ssize_t n) {   // pages, lens, free, state, page_size
  return guarded([&]() -> PyObject* {
    need_args(n, 5);
    const at::Tensor& pages = tensor_of(a[0], "pages");
    const int32_t index = device_of(pages, "pages");
    if (pages.dim() != 2) throw BadArgument("pages has to be [max_seqs, max_pages]");
    qc_table t{};
    t.max_seqs = size32(pages.size(0), "pages"), t.max_pages = size32(pages.size(1), "pages"), t.page_size = int32_of(a[4], "page_size");
    t.pages_dev = ints(a[0], "pages", index);
    t.lens_dev = ints(a[1], "lens", index, t.max_seqs);
    const at::Tensor& free = tensor_of(a[2], "free");
    t.n_pages = size32(free.numel(), "free");
    t.free_dev = ints(a[2], "free", index);
    tensor_of(a[3], "state");
    t.state_dev = ints(a[3], "state", index, 4);
    return Py_BuildValue("y#ii", reinterpret_cast<const char*>(&t), static_cast<Py_ssize_t>(sizeof t), index, t.max_seqs);
  });
}

struct Batch {
  const qc_table* table;
  int32_t index, n;
  const int32_t *ids, *count;
};

Batch batch_of(PyObject* const* a, const char* count_name) {   // packed, index, rows, counts, seq_ids, n_seqs
  Batch b{};
  char* packed = nullptr;
  Py_ssize_t size = 0;
  if (PyBytes_AsStringAndSize(a[0], &packed, &size) < 0) throw PythonError{};
  if (size != static_cast<Py_ssize_t>(sizeof(qc_table))) throw BadArgument("not a packed page table");
  b.table = reinterpret_cast<const qc_table*>(packed);
  b.index = int32_of(a[1], "device");
  const int64_t rows = int_of(a[2]);
  PyObject* listed = a[4] != Py_None ? a[4] : a[3];
  const int64_t given = a[5] == Py_None ? -1 : int_of(a[5]);
  const int64_t n = listed != Py_None ? tensor_of(listed, "seq_ids").numel() : given >= 0 ? given : rows;
  if (a[5] != Py_None && given != n) throw BadArgument("n_seqs is " + std::to_string(given) + ", but " + std::to_string(n) + " sequences are listed");
  b.n = size32(n, "n_seqs");
  b.ids = ints(a[4], "seq_ids", b.index, n);
  b.count = ints(a[3], count_name, b.index, n);
  return b;
}

PyObject* py_reset(PyObject*, PyObject* const* a, Py_ssize_t n) {   // packed, index, rows
  return guarded([&]() -> PyObject* {
    need_args(n, 3);
    PyObject* all[6] = {a[0], a[1], a[2], Py_None, Py_None, Py_None};
    const Batch b = batch_of(all, "");
    check(qc_table_reset(b.index, stream_of(b.index), b.table), "qc_table_reset");
    Py_RETURN_NONE;
  });
}

PyObject* py_extend(PyObject*, PyObject* const* a, Py_ssize_t n) {   // packed, index, rows, n_new, seq_ids, n_seqs, max_slots, lens
  return guarded([&]() -> PyObject* {
    need_args(n, 8);
    const Batch b = batch_of(a, "n_new");
    if (a[6] == Py_None && a[3] != Py_None) throw BadArgument("max_slots: the most tokens that the call may add");
    const int32_t most = a[6] == Py_None ? b.n : int32_of(a[6], "max_slots");
    if (most < 0) throw BadArgument("max_slots is negative");
    const at::Tensor& lens = tensor_of(a[7], "lens");
    if (b.n == 0) {      // (the library lists one at least; no sequence, no token)
      const auto options = at::TensorOptions().dtype(at::kInt).device(lens.device());
      return pair(at::zeros({1}, options), at::full({most}, -1, options));
    }
    const at::Tensor starts = empty({b.n + 1}, at::kInt, lens), slots = empty({most}, at::kInt, lens);
    check(qc_table_extend(b.index, stream_of(b.index), b.table, b.n, b.ids, b.count, most, starts.data_ptr<int32_t>(), most ? slots.data_ptr<int32_t>() : nullptr),
          "qc_table_extend");
    return pair(starts, slots);
  });
}

PyObject* py_trim(PyObject*, PyObject* const* a, Py_ssize_t n) {   // packed, index, rows, n_keep, seq_ids, n_seqs
  return guarded([&]() -> PyObject* {
    need_args(n, 6);
    const Batch b = batch_of(a, "n_keep");
    if (b.n == 0) Py_RETURN_NONE;
    check(qc_table_trim(b.index, stream_of(b.index), b.table, b.n, b.ids, b.count), "qc_table_trim");
    Py_RETURN_NONE;
  });
}

// ---- rows -----------------------------------------------------------------------------------------------------

int64_t page_row(int64_t heads, int64_t page, int64_t head_dim) { return heads * page * (head_dim / 2 + 4); }

PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) {   // k_pool, v_pool, slots, k, v, page_size
  return guarded([&]() -> PyObject* {
    need_args(n, 6);
    const bool has_k = a[3] != Py_None, has_v = a[4] != Py_None;
    if ((!has_k && !has_v) || has_k != (a[0] != Py_None) || has_v != (a[1] != Py_None)) throw BadArgument("a pool for every tensor, and one of k and v at least");
    const at::Tensor& rows = tensor_of(has_k ? a[3] : a[4], has_k ? "k" : "v");
    const int32_t index = device_of(rows, has_k ? "k" : "v");
    if (rows.dim() != 3) throw BadArgument("k and v have to be [tokens, heads, head_dim]");
    const int32_t page = int32_of(a[5], "page_size");
    const int64_t row = page_row(rows.size(1), page, rows.size(2));
    const void *k = nullptr, *v = nullptr;
    void *kp = nullptr, *vp = nullptr;
    int64_t ks = 0, vs = 0;
    if (has_k) ks = rows_of(rows, "k", index), k = rows.data_ptr(), kp = pool_of(tensor_of(a[0], "k_pool"), "k_pool", row, index);
    if (has_v) {
      const at::Tensor& t = tensor_of(a[4], "v");
      vs = rows_of(t, "v", index), v = t.data_ptr(), vp = pool_of(tensor_of(a[1], "v_pool"), "v_pool", row, index);
      if (has_k && (t.sizes() != rows.sizes() || THPVariable_Unpack(a[0]).sizes() != THPVariable_Unpack(a[1]).sizes()))
        throw BadArgument("k and v, and their pools, have to have the same shape");
    }
    const qc_quant_shape shape{size32(rows.size(1), "heads"), size32(rows.size(2), "head_dim"), page, size32(THPVariable_Unpack(has_k ? a[0] : a[1]).size(0), "pages")};
    tensor_of(a[2], "slots");
    const int32_t* slots = ints(a[2], "slots", index, rows.size(0));
    if (rows.size(0)) check(qc_quant_append(index, stream_of(index), &shape, size32(rows.size(0), "tokens"), slots, k, ks, v, vs, kp, vp), "qc_quant_append");
    Py_RETURN_NONE;
  });
}

at::Tensor out_of(PyObject* o, at::IntArrayRef sizes, const at::Tensor& like, const char* name, int32_t index, bool zero) {
  if (o == Py_None) return zero ? at::zeros(sizes, at::TensorOptions().dtype(at::kBFloat16).device(like.device())) : empty(sizes, at::kBFloat16, like);
  const at::Tensor& t = tensor_of(o, name);
  if (t.sizes() != sizes || t.scalar_type() != at::kBFloat16 || !on(t, index) || !t.is_contiguous()) {
    std::string s;
    for (const int64_t x : sizes) s += (s.empty() ? "" : ", ") + std::to_string(x);
    throw BadArgument(std::string(name) + " has to be a dense bfloat16 tensor [" + s + "] on " + cuda_name(index));
  }
  return t;
}

PyObject* py_read(PyObject*, PyObject* const* a, Py_ssize_t n) {   // k_pool, v_pool, slots, heads, head_dim, page_size, k_out, v_out
  return guarded([&]() -> PyObject* {
    need_args(n, 8);
    const at::Tensor& slots = tensor_of(a[2], "slots");
    const int32_t index = device_of(slots, "slots");
    const bool has_k = a[0] != Py_None, has_v = a[1] != Py_None;
    if (!has_k && !has_v) throw BadArgument("one of k_pool and v_pool at least");
    qc_quant_shape shape{int32_of(a[3], "n_kv_heads"), int32_of(a[4], "head_dim"), int32_of(a[5], "page_size"), 0};
    const int64_t tokens = slots.numel(), row = page_row(shape.n_kv_heads, shape.page_size, shape.head_dim);
    if (shape.n_kv_heads < 0 || shape.head_dim < 0) throw BadArgument("n_kv_heads and head_dim are sizes");
    const int64_t sizes[3] = {tokens, shape.n_kv_heads, shape.head_dim};
    const void *kp = nullptr, *vp = nullptr;
    at::Tensor k, v;
    if (has_k) kp = pool_of(tensor_of(a[0], "k_pool"), "k_pool", row, index), k = out_of(a[6], sizes, slots, "k_out", index, true);
    if (has_v) vp = pool_of(tensor_of(a[1], "v_pool"), "v_pool", row, index), v = out_of(a[7], sizes, slots, "v_out", index, true);
    if (has_k && has_v && THPVariable_Unpack(a[0]).size(0) != THPVariable_Unpack(a[1]).size(0)) throw BadArgument("the pools have to have the same shape");
    shape.n_pages = size32(THPVariable_Unpack(has_k ? a[0] : a[1]).size(0), "pages");
    const int32_t* at = ints(a[2], "slots", index);
    if (tokens)
      check(qc_quant_read(index, stream_of(index), &shape, size32(tokens, "tokens"), at, kp, vp, has_k ? k.data_ptr() : nullptr, has_v ? v.data_ptr() : nullptr),
            "qc_quant_read");
    if (has_k && has_v) return pair(k, v);
    PyObject* one = THPVariable_Wrap(has_k ? k : v);
    if (!one) throw PythonError{};
    return has_k ? Py_BuildValue("NO", one, Py_None) : Py_BuildValue("ON", Py_None, one);
  });
}

// ---- attention --------------------------------------------------------------------------------------------------

qc_quant_stream stream_args(PyObject* o, const char* name, int64_t row, at::IntArrayRef sizes, int64_t rows, int32_t index) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 5) throw BadArgument(std::string(name) + " has to be a Stream");
  const std::string at = name;
  const at::Tensor& q = tensor_of(PyTuple_GET_ITEM(o, 0), (at + ".q").c_str());
  const at::Tensor& k = tensor_of(PyTuple_GET_ITEM(o, 1), (at + ".k_pool").c_str());
  const at::Tensor& v = tensor_of(PyTuple_GET_ITEM(o, 2), (at + ".v_pool").c_str());
  const at::Tensor& pages = tensor_of(PyTuple_GET_ITEM(o, 3), (at + ".pages").c_str());
  tensor_of(PyTuple_GET_ITEM(o, 4), (at + ".lens").c_str());
  qc_quant_stream s{};
  s.q_stride = rows_of(q, (at + ".q").c_str(), index);
  if (q.sizes() != sizes) throw BadArgument(at + ".q has to have the shape of the text stream's");
  if (pages.dim() != 2 || (rows >= 0 && pages.size(0) != rows)) throw BadArgument(at + ".pages has to be [sequences, pages], with as many rows as the other stream's");
  s.q_dev = q.data_ptr();
  s.k_pool_dev = pool_of(k, (at + ".k_pool").c_str(), row, index), s.v_pool_dev = pool_of(v, (at + ".v_pool").c_str(), row, index);
  if (k.size(0) != v.size(0)) throw BadArgument(at + ": the pools have to have the same shape");
  s.pages_dev = ints(PyTuple_GET_ITEM(o, 3), (at + ".pages").c_str(), index);
  s.lens_dev = ints(PyTuple_GET_ITEM(o, 4), (at + ".lens").c_str(), index, pages.size(0));
  s.max_pages = size32(pages.size(1), "pages"), s.n_pages = size32(k.size(0), "pages");
  return s;
}

// text, n_kv_heads, page_size, visual, seq_ids, starts, max_queries, causal, scale, out, status
PyObject* py_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need_args(n, 11);
    if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 5) throw BadArgument("text has to be a Stream");
    const at::Tensor& q = tensor_of(PyTuple_GET_ITEM(a[0], 0), "text.q");
    const int32_t index = device_of(q, "text.q");
    if (q.dim() != 3) throw BadArgument("text.q has to be [tokens, heads, head_dim]");
    qc_quant_attend_args args{};
    args.n_q_heads = size32(q.size(1), "heads"), args.head_dim = size32(q.size(2), "head_dim"), args.n_tokens = size32(q.size(0), "tokens");
    args.n_kv_heads = int32_of(a[1], "n_kv_heads"), args.page_size = int32_of(a[2], "page_size"), args.max_queries = int32_of(a[6], "max_queries");
    const int64_t row = page_row(args.n_kv_heads, args.page_size, args.head_dim);
    args.text = stream_args(a[0], "text", row, q.sizes(), -1, index);
    const int64_t rows = THPVariable_Unpack(PyTuple_GET_ITEM(a[0], 3)).size(0);
    args.max_seqs = size32(rows, "pages");
    if (a[3] != Py_None) args.visual = stream_args(a[3], "visual", row, q.sizes(), rows, index);
    int64_t seqs = q.size(0);
    if (a[4] != Py_None) seqs = tensor_of(a[4], "seq_ids").numel();
    else if (a[5] != Py_None) seqs = tensor_of(a[5], "starts").numel() - 1;
    args.n_seqs = size32(seqs, "seq_ids");
    args.seq_ids_dev = ints(a[4], "seq_ids", index, seqs), args.starts_dev = ints(a[5], "starts", index, seqs + 1), args.status_dev = ints(a[10], "status", index, 1);
    const int causal = PyObject_IsTrue(a[7]);
    if (causal < 0) throw PythonError{};
    args.causal = causal;
    const double scale = PyFloat_AsDouble(a[8]);
    if (scale == -1.0 && PyErr_Occurred()) throw PythonError{};
    args.softmax_scale = static_cast<float>(scale);
    const at::Tensor out = out_of(a[9], q.sizes(), q, "out", index, false), lse = empty({q.size(0), q.size(1)}, at::kFloat, q);
    if (q.size(0) && seqs) {
      check(qc_quant_workspace_bytes(&args, &args.workspace_bytes), "qc_quant_attend");
      const at::Tensor workspace = empty({static_cast<int64_t>(args.workspace_bytes)}, at::kByte, q);   // the call's own, back to the allocator behind it
      args.out_dev = out.data_ptr(), args.lse_out_dev = lse.data_ptr<float>(), args.workspace_dev = workspace.data_ptr();
      check(qc_quant_attend(index, stream_of(index), &args), "qc_quant_attend");
    }
    return pair(out, lse);
  });
}

PyObject* py_error_class(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need_args(n, 1);
    Py_INCREF(a[0]);
    Py_XSETREF(g_qc_error, a[0]);
    Py_RETURN_NONE;
  });
}

PyMethodDef g_methods[] = {
    {"table", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_table)), METH_FASTCALL, nullptr},
    {"reset", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_reset)), METH_FASTCALL, nullptr},
    {"extend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_extend)), METH_FASTCALL, nullptr},
    {"trim", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_trim)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_append)), METH_FASTCALL, nullptr},
    {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_read)), METH_FASTCALL, nullptr},
    {"attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_attend)), METH_FASTCALL, nullptr},
    {"error_class", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_error_class)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
#ifndef QC_BUILT_FOR
#define QC_BUILT_FOR "an unknown torch"
#endif
const char g_built_for[] = "_qc_torch for " QC_BUILT_FOR ";";      // (build.py looks for it in the file)

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_qc_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qc_torch() {
  PyObject* m = PyModule_Create(&g_module);
  if (m && PyModule_AddStringConstant(m, "built_for", g_built_for) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
