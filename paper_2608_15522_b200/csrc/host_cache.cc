// Whole calls of the paged cache for the wrappers of binding.py: tensors are checked and read, what the caller did not bring is allocated,
// and the library is called, without the interpreter lock from the first allocation on (an allocation may wait for the GPU).
// One native call each, because a token's step is short: its attention takes 10 us on the device.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <torch/csrc/utils/object_ptr.h>

#include <climits>

#include "../../include/avsa.h"

namespace {

decltype(&avsa_prefix_attn_step) f_attn;
decltype(&avsa_prefix_attn_workspace_bytes) f_attn_ws;
decltype(&avsa_cache_extend_step) f_extend;
decltype(&avsa_cache_write) f_write;
decltype(&avsa_cache_fork_step) f_fork;
decltype(&avsa_cache_free_step) f_free;
decltype(&avsa_cache_compact_step) f_compact;
decltype(&avsa_cache_workspace_bytes) f_ws;
PyObject* o_raw_stream;

template <typename F>
void without_lock(F&& work) {
  struct Lock {
    PyThreadState* state = PyEval_SaveThread();
    ~Lock() { PyEval_RestoreThread(state); }
  } lock;
  work();
}

// A tensor argument, held for the length of the call.  Everything about it is read once, with the interpreter lock: another thread may change
// the caller's tensor meanwhile.
struct Arg {
  at::Tensor t;
  void* ptr = nullptr;
  int64_t numel = 0;
  bool there() const { return t.defined(); }
  template <typename T>
  T* as() const { return static_cast<T*>(ptr); }
};

struct Call {
  PyObject* const* a;
  at::Device device = at::Device(at::kCPU);
  void* stream = nullptr;

  const at::Tensor& tensor(int i, const char* name) {
    TORCH_CHECK_TYPE(THPVariable_Check(a[i]), name, ": expected a tensor");
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    TORCH_CHECK_VALUE(t.is_cuda() && t.layout() == at::kStrided, name, ": expected a tensor on a CUDA device");
    if (!device.is_cuda()) device = t.device();
    TORCH_CHECK_VALUE(t.device() == device, name, ": on another device than the call's first tensor");
    return t;
  }
  // contiguous, of a type and a number of dimensions (0: any); None only where it may be
  Arg plain(int i, const char* name, at::ScalarType type, int64_t dims, bool optional = false) {
    Arg r;
    if (optional && a[i] == Py_None) return r;
    const at::Tensor& t = tensor(i, name);
    TORCH_CHECK_VALUE(t.scalar_type() == type, name, ": expected ", at::toString(type), ", got ", at::toString(t.scalar_type()));
    TORCH_CHECK_VALUE(dims == 0 || t.dim() == dims, name, ": expected ", dims, " dimensions, got ", t.dim());
    TORCH_CHECK_VALUE(t.is_contiguous(), name, ": expected a contiguous tensor");
    r.t = t;
    r.ptr = t.data_ptr();
    r.numel = t.numel();
    return r;
  }
  Arg ints(int i, const char* name, int64_t dims, bool optional = false) { return plain(i, name, at::kInt, dims, optional); }
  // the record of the first error of many calls
  Arg log(int i) {
    const Arg r = ints(i, "log", 1, true);
    TORCH_CHECK_VALUE(!r.there() || r.numel == 4, "log: expected four entries");
    return r;
  }
  bool flag(int i, const char* name) {
    TORCH_CHECK_TYPE(PyBool_Check(a[i]), name, ": expected a bool");
    return a[i] == Py_True;
  }
  int integer(int i, const char* name) {
    TORCH_CHECK_TYPE(PyLong_Check(a[i]) && !PyBool_Check(a[i]), name, ": expected an int");
    int overflow;
    const long v = PyLong_AsLongAndOverflow(a[i], &overflow);
    TORCH_CHECK_VALUE(overflow == 0 && v >= INT_MIN && v <= INT_MAX, name, ": out of range");
    return static_cast<int>(v);
  }
  float number(int i, const char* name) {
    const double v = PyFloat_AsDouble(a[i]);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return static_cast<float>(v);
  }
  // the current stream of the call's device; behind the last tensor
  void find_stream() {
    THPObjectPtr index(PyLong_FromLong(device.index()));
    if (!index) throw python_error();
    THPObjectPtr raw(PyObject_CallOneArg(o_raw_stream, index.get()));
    if (!raw) throw python_error();
    stream = PyLong_AsVoidPtr(raw.get());
    if (stream == nullptr && PyErr_Occurred()) throw python_error();
  }
  void make(Arg& r, at::ScalarType type, at::IntArrayRef sizes) const {
    if (r.there()) return;
    r.t = at::empty(sizes, at::TensorOptions().dtype(type).device(device));
    r.ptr = r.t.data_ptr();
    r.numel = r.t.numel();
  }
  void make_ws(Arg& r, size_t bytes) const { make(r, at::kByte, {static_cast<int64_t>(bytes > 256 ? bytes : 256)}); }
  // the caller's own object where there was one
  PyObject* give(int i, const Arg& r) const { return a[i] != Py_None ? Py_NewRef(a[i]) : r.there() ? THPVariable_Wrap(r.t) : Py_NewRef(Py_None); }
};

int size32(const at::Tensor& t, int i) {
  const int64_t n = t.size(i);
  TORCH_CHECK_VALUE(n <= INT_MAX, "a dimension beyond 32 bits");
  return static_cast<int>(n);
}

// bf16 of four dimensions with a contiguous last one
struct View : Arg {
  int64_t size[4], stride[4];
  operator avsa_bf16_4d() const { return avsa_bf16_4d{ptr, stride[0], stride[1], stride[2]}; }
  int dim(int i) const { return static_cast<int>(size[i]); }
};
View take_view(Call& c, int i, const char* name) {
  const at::Tensor& t = c.tensor(i, name);
  TORCH_CHECK_VALUE(t.scalar_type() == at::kBFloat16 && t.dim() == 4, name, ": expected a bf16 tensor of four dimensions");
  TORCH_CHECK_VALUE(t.size(3) <= 1 || t.stride(3) == 1, name, ": the head dimension must be contiguous");
  View r;
  for (int k = 0; k < 4; k++) {
    r.size[k] = size32(t, k);
    r.stride[k] = t.stride(k);
  }
  r.t = t;
  r.ptr = t.data_ptr();
  r.numel = t.numel();
  return r;
}

PyObject* result(int status, std::initializer_list<PyObject*> items) {
  PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(items.size()) + 1);
  PyObject* st = PyLong_FromLong(status);
  bool ok = r != nullptr && st != nullptr;
  for (PyObject* i : items) ok = ok && i != nullptr;
  if (!ok) {
    Py_XDECREF(r);
    Py_XDECREF(st);
    for (PyObject* i : items) Py_XDECREF(i);
    return nullptr;
  }
  PyTuple_SET_ITEM(r, 0, st);
  Py_ssize_t at = 1;
  for (PyObject* i : items) PyTuple_SET_ITEM(r, at++, i);
  return r;
}

void arity(Py_ssize_t got, Py_ssize_t want) {
  TORCH_CHECK_TYPE(got == want && f_attn != nullptr, "wrong number of arguments, or bind() has not been called");
}

// attn(q, k_pool, v_pool, table, length, prefix_pages, seq, causal, softmax_scale, want_lse, o, lse, ws, count, log) -> (status, o, lse, ws)
PyObject* py_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 15);
  Call c{a};
  const View q = take_view(c, 0, "q"), k = take_view(c, 1, "k_pool"), v = take_view(c, 2, "v_pool");
  const Arg table = c.ints(3, "table", 2), length = c.ints(4, "length", 1);
  const int prefix_pages = c.integer(5, "prefix_pages");
  const Arg seq = c.ints(6, "seq", 1, true);
  const bool causal = c.flag(7, "causal");
  const float scale = c.number(8, "softmax_scale");
  const bool want_lse = c.flag(9, "want_lse");
  const int B = q.dim(0), H = q.dim(1), L = q.dim(2), d = q.dim(3), pages = k.dim(0), Hkv = k.dim(1), page = k.dim(2);
  const int seqs = size32(table.t, 0), width = size32(table.t, 1);
  for (int i = 0; i < 4; i++) TORCH_CHECK_VALUE(k.size[i] == v.size[i], "k_pool and v_pool have different shapes");
  TORCH_CHECK_VALUE(k.dim(3) == d, "q and the pools have different head dimensions");
  TORCH_CHECK_VALUE(length.numel == seqs, "length: one entry for each row of the table");
  TORCH_CHECK_VALUE(seq.there() ? seq.numel == B : B <= seqs, "q has more batch entries than there are sequences");
  Arg o, lse;
  if (a[10] != Py_None) {
    const View given = take_view(c, 10, "o");
    for (int i = 0; i < 4; i++)
      TORCH_CHECK_VALUE(given.size[i] == q.size[i] && (q.size[i] <= 1 || given.stride[i] == q.stride[i]), "o: expected the shape and strides of q");
    o = given;
  }
  if (want_lse) {
    lse = c.plain(11, "lse", at::kFloat, 3, true);
    TORCH_CHECK_VALUE(!lse.there() || lse.numel == static_cast<int64_t>(B) * H * L, "lse: expected [B,H,L]");
  }
  Arg ws = c.plain(12, "ws", at::kByte, 1, true);
  const Arg count = c.ints(13, "count", 1, true);
  TORCH_CHECK_VALUE(!count.there() || count.numel == B, "count: one entry for each batch entry of q");
  const Arg log = c.log(14);
  c.find_stream();
  int st;
  without_lock([&] {
    if (!o.there()) {
      o.t = at::empty_strided(q.size, q.stride, at::TensorOptions().dtype(at::kBFloat16).device(c.device));
      o.ptr = o.t.data_ptr();
    }
    if (want_lse) c.make(lse, at::kFloat, {B, H, L});
    if (!ws.there()) c.make_ws(ws, f_attn_ws(B, H, Hkv, L, d, page, width, prefix_pages));
    st = f_attn(B, H, Hkv, L, d, page, pages, seqs, width, q, k, v, table.as<int32_t>(), length.as<int32_t>(), seq.as<int32_t>(),
                count.as<int32_t>(), prefix_pages, causal ? AVSA_CAUSAL : 0u, scale, o.ptr, lse.as<float>(), log.as<int32_t>(), ws.ptr,
                static_cast<size_t>(ws.numel), c.stream);
  });
  return result(st, {c.give(10, o), c.give(11, lse), c.give(12, ws)});
  END_HANDLE_TH_ERRORS
}

// The state of a cache at arguments [at, at + 3), and the arrays that the state behind the call goes to at [to, to + 3) (None: the same).
struct State {
  Arg table, length, ref, table_out, length_out, ref_out;
  State(Call& c, int at, int to)
      : table(c.ints(at, "table", 2)), length(c.ints(at + 1, "length", 1)), ref(c.ints(at + 2, "ref", 1)),
        table_out(c.ints(to, "table (out)", 2, true)), length_out(c.ints(to + 1, "length (out)", 1, true)),
        ref_out(c.ints(to + 2, "ref (out)", 1, true)) {
    TORCH_CHECK_VALUE(length.numel == table.t.size(0), "length: one entry for each row of the table");
    if (!table_out.there()) table_out = table;
    if (!length_out.there()) length_out = length;
    if (!ref_out.there()) ref_out = ref;
    TORCH_CHECK_VALUE(table_out.t.sizes() == table.t.sizes() && length_out.numel == length.numel && ref_out.numel == ref.numel,
                      "out: expected the shapes of table, length and ref");
  }
  avsa_cache cache(int page) const {
    return avsa_cache{table.as<int32_t>(), length.as<int32_t>(), ref.as<int32_t>(), table_out.as<int32_t>(), length_out.as<int32_t>(),
                      ref_out.as<int32_t>(), size32(table.t, 0), size32(table.t, 1), size32(ref.t, 0), page};
  }
};
PyObject* wrap(const Arg& r) { return THPVariable_Wrap(r.t); }

// bf16 [planes,pages,Hkv,page,d], a page of a plane in one piece, its heads or its tokens outermost
avsa_pages take_pool(Call& c, int i, int64_t pages, int* page, Arg& hold) {
  const at::Tensor& t = c.tensor(i, "pool");
  TORCH_CHECK_VALUE(t.scalar_type() == at::kBFloat16 && t.dim() == 5, "pool: expected a bf16 tensor [planes,pages,Hkv,page,d]");
  TORCH_CHECK_VALUE(t.size(1) == pages, "pool: as many pages as ref has entries");
  const int64_t h = t.size(2), p = t.size(3), d = t.size(4), sh = t.stride(2), sp = t.stride(3);
  const bool heads_out = (h <= 1 || sh == p * d) && (p <= 1 || sp == d), tokens_out = (p <= 1 || sp == h * d) && (h <= 1 || sh == d);
  TORCH_CHECK_VALUE((d <= 1 || t.stride(4) == 1) && (heads_out || tokens_out), "pool: a page has to be in one piece");
  *page = size32(t, 3);
  hold.t = t;
  hold.ptr = t.data_ptr();
  return avsa_pages{hold.ptr, size32(t, 0), h * p * d * 2, t.stride(0) * 2, t.stride(1) * 2};
}

int list_size(const Arg& x, const Arg& y, const char* text) {
  TORCH_CHECK_VALUE(x.numel == y.numel && x.numel <= INT_MAX, text);
  return static_cast<int>(x.numel);
}

// extend(table, length, ref, seq, count, page, table_out, length_out, ref_out, ws, granted, log) -> (status, table, length, ref, ws)
PyObject* py_extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 12);
  Call c{a};
  const State s(c, 0, 6);
  const Arg seq = c.ints(3, "seq", 1), count = c.ints(4, "count", 1);
  const int entries = list_size(seq, count, "seq and count have different lengths");
  const avsa_cache cache = s.cache(c.integer(5, "page"));
  Arg ws = c.plain(9, "ws", at::kByte, 1, true);
  const Arg granted = c.ints(10, "granted", 1, true);
  TORCH_CHECK_VALUE(!granted.there() || granted.numel == entries, "granted: one entry for each of seq");
  const Arg log = c.log(11);
  c.find_stream();
  int st;
  without_lock([&] {
    if (!ws.there()) c.make_ws(ws, f_ws(cache.seqs, cache.pages, entries));
    st = f_extend(cache, seq.as<int32_t>(), count.as<int32_t>(), entries, granted.as<int32_t>(), log.as<int32_t>(), ws.ptr,
                  static_cast<size_t>(ws.numel), c.stream);
  });
  return result(st, {wrap(s.table_out), wrap(s.length_out), wrap(s.ref_out), c.give(9, ws)});
  END_HANDLE_TH_ERRORS
}

// write(k_new, v_new, k_pool, v_pool, table, length, seq, count) -> status
PyObject* py_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 8);
  Call c{a};
  const View kn = take_view(c, 0, "k_new"), vn = take_view(c, 1, "v_new"), k = take_view(c, 2, "k_pool"), v = take_view(c, 3, "v_pool");
  const Arg table = c.ints(4, "table", 2), length = c.ints(5, "length", 1), seq = c.ints(6, "seq", 1, true), count = c.ints(7, "count", 1, true);
  const int seqs = size32(table.t, 0), width = size32(table.t, 1), entries = kn.dim(0);
  for (int i = 0; i < 4; i++)
    TORCH_CHECK_VALUE(kn.size[i] == vn.size[i] && k.size[i] == v.size[i], "keys and values have different shapes");
  TORCH_CHECK_VALUE(kn.dim(1) == k.dim(1) && kn.dim(3) == k.dim(3), "the new tokens and the pools have different heads");
  TORCH_CHECK_VALUE(length.numel == seqs, "length: one entry for each row of the table");
  TORCH_CHECK_VALUE((seq.there() ? seq.numel == entries : entries <= seqs) && (!count.there() || count.numel == entries),
                    "seq and count: one entry for each of the new tokens' batch entries");
  c.find_stream();
  int st;
  without_lock([&] {
    st = f_write(entries, kn.dim(1), kn.dim(2), kn.dim(3), k.dim(2), k.dim(0), seqs, width, kn, vn, k, v, table.as<int32_t>(), length.as<int32_t>(),
                 seq.as<int32_t>(), count.as<int32_t>(), c.stream);
  });
  return PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// fork(pool, table, length, ref, parent, child, table_out, length_out, ref_out, ws, log) -> (status, table, length, ref, ws)
PyObject* py_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 11);
  Call c{a};
  const State s(c, 1, 6);
  Arg hold;
  int page;
  const avsa_pages pool = take_pool(c, 0, s.ref.numel, &page, hold);
  const Arg parent = c.ints(4, "parent", 1), child = c.ints(5, "child", 1);
  const int entries = list_size(parent, child, "parent and child have different lengths");
  const avsa_cache cache = s.cache(page);
  Arg ws = c.plain(9, "ws", at::kByte, 1, true);
  const Arg log = c.log(10);
  c.find_stream();
  int st;
  without_lock([&] {
    if (!ws.there()) c.make_ws(ws, f_ws(cache.seqs, cache.pages, entries));
    st = f_fork(cache, pool, parent.as<int32_t>(), child.as<int32_t>(), entries, log.as<int32_t>(), ws.ptr, static_cast<size_t>(ws.numel), c.stream);
  });
  return result(st, {wrap(s.table_out), wrap(s.length_out), wrap(s.ref_out), c.give(9, ws)});
  END_HANDLE_TH_ERRORS
}

// free(table, length, ref, seq, table_out, length_out, ref_out, ws, log) -> (status, table, length, ref, ws)
PyObject* py_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 9);
  Call c{a};
  const State s(c, 0, 4);
  const Arg seq = c.ints(3, "seq", 1);
  const int entries = list_size(seq, seq, "seq");
  const avsa_cache cache = s.cache(0);
  Arg ws = c.plain(7, "ws", at::kByte, 1, true);
  const Arg log = c.log(8);
  c.find_stream();
  int st;
  without_lock([&] {
    if (!ws.there()) c.make_ws(ws, f_ws(cache.seqs, cache.pages, entries));
    st = f_free(cache, seq.as<int32_t>(), entries, log.as<int32_t>(), ws.ptr, static_cast<size_t>(ws.numel), c.stream);
  });
  return result(st, {wrap(s.table_out), wrap(s.length_out), wrap(s.ref_out), c.give(7, ws)});
  END_HANDLE_TH_ERRORS
}

// compact(pool, table, length, ref, table_out, length_out, ref_out, n_live, ws, log) -> (status, n_live, ws)
PyObject* py_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 10);
  Call c{a};
  const State s(c, 1, 4);
  Arg hold;
  int page;
  const avsa_pages pool = take_pool(c, 0, s.ref.numel, &page, hold);
  const avsa_cache cache = s.cache(page);
  Arg n_live = c.ints(7, "n_live", 1, true), ws = c.plain(8, "ws", at::kByte, 1, true);
  const Arg log = c.log(9);
  TORCH_CHECK_VALUE(!n_live.there() || n_live.numel >= 1, "n_live: expected one entry");
  c.find_stream();
  int st;
  without_lock([&] {
    c.make(n_live, at::kInt, {1});
    if (!ws.there()) c.make_ws(ws, f_ws(cache.seqs, cache.pages, 0));
    st = f_compact(cache, pool, n_live.as<int32_t>(), log.as<int32_t>(), ws.ptr, static_cast<size_t>(ws.numel), c.stream);
  });
  return result(st, {c.give(7, n_live), c.give(8, ws)});
  END_HANDLE_TH_ERRORS
}

// bind(addresses of prefix_attn, its workspace query, extend, write, fork, free, compact, the cache's workspace query; reader of the raw current stream)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 9, "wrong number of arguments");
  void* p[8];
  for (int i = 0; i < 8; i++) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (p[i] == nullptr) {
      TORCH_CHECK_VALUE(PyErr_Occurred(), "a null address");
      return nullptr;
    }
  }
  o_raw_stream = Py_NewRef(a[8]);
  f_attn = reinterpret_cast<decltype(f_attn)>(p[0]);
  f_attn_ws = reinterpret_cast<decltype(f_attn_ws)>(p[1]);
  f_extend = reinterpret_cast<decltype(f_extend)>(p[2]);
  f_write = reinterpret_cast<decltype(f_write)>(p[3]);
  f_fork = reinterpret_cast<decltype(f_fork)>(p[4]);
  f_free = reinterpret_cast<decltype(f_free)>(p[5]);
  f_compact = reinterpret_cast<decltype(f_compact)>(p[6]);
  f_ws = reinterpret_cast<decltype(f_ws)>(p[7]);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_bind)), METH_FASTCALL, nullptr},
    {"attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_attn)), METH_FASTCALL, nullptr},
    {"extend", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_extend)), METH_FASTCALL, nullptr},
    {"write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_write)), METH_FASTCALL, nullptr},
    {"fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_fork)), METH_FASTCALL, nullptr},
    {"free", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_free)), METH_FASTCALL, nullptr},
    {"compact", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(py_compact)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_avsa_cache", "whole calls of the paged cache", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__avsa_cache(void) { return PyModule_Create(&module); }
