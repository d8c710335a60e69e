// The calls of a small problem from Python without the cost of marshalling them in Python: dfs_forward, the token orders and the staged calls
// of a quality check take their arguments straight from the objects.  A launch costs the host some 3 us and its kernel often less, so what bounds
// such calls is what Python does between two of them: some fifty attribute lookups of tensors and a ctypes call.  Measured (us, in Python ->
// here).  The host's time of a call in a burst of eight: refresh and reuse step of 256 fp32 tokens (one launch each) 9.7 -> 4.7 and 9.9 -> 5.0, token
// order 6.4 -> 3.9.  A call among others: token order of 75 600 or 64 tokens 6.2 -> 3.6, reuse step of 512 tokens x 8 heads, d = 64,
// 9.4 -> 7.3, of 256 fp32 tokens 9.2 -> 8.7; the refresh step of these stays at 12.4, which its kernel takes.
// A quality check in staged calls (nine of them and two of torch), 675 tokens x 2 heads, d = 64, 73 -> 53, 1 575 x 2 73 -> 62; larger ones
// take what their kernels take (2 625 x 4, d = 128, 111).
//
// The module holds the version of the torch it was built against, whose classes it reads: binding.py uses it with no other.
// A call goes to the library only if every argument is of the plain kind and passes every check of binding.py; else None is returned,
// nothing has happened, and binding.py does the call, or raises, in its own way.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPStream.h>

#include <cstring>

#include "../../include/dfsattn.h"

namespace {

// binding.Geom, QkGeom, Window, Packed and Paged, ctypes structures with the layouts of dfs_geom, dfs_qk_geom, dfs_window, dfs_packed and
// dfs_paged
PyObject *g_geom_type = nullptr, *g_qk_type = nullptr, *g_window_type = nullptr, *g_packed_type = nullptr, *g_paged_type = nullptr;
PyObject *s_kv_idx, *s_kv_cnt, *s_mask, *s_k_head, *s_K_max;
PyObject *s_k, *s_v, *s_table, *s_k_scale, *s_v_scale;

struct NotPlain {};                                 // thrown where binding.py has to look at an argument

void need(bool ok) {
  if (!ok) throw NotPlain();
}

int to_int(PyObject* x) {
  need(PyLong_CheckExact(x));
  int overflow = 0;
  const long v = PyLong_AsLongAndOverflow(x, &overflow);
  need(!overflow && v == long(int(v)));
  return int(v);
}

double to_double(PyObject* x) {
  if (PyFloat_CheckExact(x)) return PyFloat_AS_DOUBLE(x);
  return double(to_int(x));
}

template <class S>
S to_struct(PyObject* x, PyObject* type) {
  need(reinterpret_cast<PyObject*>(Py_TYPE(x)) == type);
  S s;
  Py_buffer b;
  need(PyObject_GetBuffer(x, &b, PyBUF_SIMPLE) == 0);
  const bool fits = b.len == Py_ssize_t(sizeof(s));
  if (fits) std::memcpy(&s, b.buf, sizeof(s));
  PyBuffer_Release(&b);
  need(fits);
  return s;
}
dfs_geom to_geom(PyObject* x) { return to_struct<dfs_geom>(x, g_geom_type); }

// A contiguous device tensor of at least `numel` elements (of `type`, if one is given): its address.
void* to_ptr(PyObject* x, at::ScalarType type, int64_t numel, int64_t* bytes = nullptr) {
  need(THPVariable_CheckExact(x));
  const at::Tensor& t = THPVariable_Unpack(x);
  need(t.is_cuda() && t.is_contiguous() && (type == at::ScalarType::Undefined || t.scalar_type() == type) && t.numel() >= numel);
  if (bytes) *bytes = t.numel() * int64_t(t.element_size());
  return t.data_ptr();
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

struct Attr {                                       // an attribute, held while its address is in use
  PyObject* o;
  Attr(PyObject* from, PyObject* name) : o(PyObject_GetAttr(from, name)) { need(o != nullptr); }
  ~Attr() { Py_XDECREF(o); }
  Attr(const Attr&) = delete;
  void* ptr(at::ScalarType type, int64_t numel) const { return o == Py_None ? nullptr : to_ptr(o, type, numel); }
};

// Runs a call; None if an argument is not plain, else the library's status.
template <class F>
PyObject* guarded(F f) {
  int rc;
  try {
    rc = f();
  } catch (...) {                                   // NotPlain, or what torch throws about a tensor without memory
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  return PyLong_FromLong(rc);
}

PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 15);
    const dfs_geom g = to_geom(a[0]);
    dfs_sizes s;
    need(dfs_geom_sizes(&g, &s) == DFS_OK);
    const int dtype = to_int(a[1]), mode = to_int(a[8]), refresh = PyObject_IsTrue(a[7]);
    need(refresh >= 0);
    const auto type = dtype == DFS_BF16 ? at::kBFloat16 : at::kFloat;
    const int64_t numel = int64_t(g.heads) * s.N * g.d, rows = int64_t(g.heads) * s.M;
    PyObject* st = a[11];
    const Attr kv_idx(st, s_kv_idx), kv_cnt(st, s_kv_cnt), mask(st, s_mask), k_head(st, s_k_head), K_max(st, s_K_max);
    dfs_mask_state m;
    m.K_max = to_int(K_max.o);
    m.kv_idx = static_cast<int32_t*>(kv_idx.ptr(at::kInt, rows * m.K_max));
    m.kv_cnt = static_cast<int32_t*>(kv_cnt.ptr(at::kInt, rows));
    m.mask = static_cast<uint8_t*>(mask.ptr(at::kByte, rows * s.M));
    m.k_head = static_cast<int32_t*>(k_head.ptr(at::kInt, g.heads));
    const void *q = to_ptr(a[2], type, numel), *k = to_ptr(a[3], type, numel), *v = to_ptr(a[4], type, numel);
    const auto* perm_pad = static_cast<const int32_t*>(to_ptr(a[5], at::kInt, s.N_pad));
    const auto* inv = static_cast<const int32_t*>(to_ptr(a[6], at::kInt, s.N));
    const double sparsity = to_double(a[9]), mass = to_double(a[10]);
    const float scale = float(to_double(a[12]));
    void* o = to_ptr(a[13], type, numel);
    int64_t ws_bytes = 0;
    void* ws = to_ptr(a[14], at::ScalarType::Undefined, 0, &ws_bytes);
    void* st_ = stream();
    PyThreadState* gil = PyEval_SaveThread();
    const int rc = dfs_forward(&g, dtype, q, k, v, perm_pad, inv, refresh, mode, sparsity, mass, &m, scale, o, ws, size_t(ws_bytes), st_);
    PyEval_RestoreThread(gil);
    return rc;
  });
}

PyObject* token_order(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 6);
    const dfs_geom g = to_geom(a[0]);
    dfs_sizes s;
    need(dfs_geom_sizes(&g, &s) == DFS_OK);
    const int order = to_int(a[1]);
    auto* perm_pad = static_cast<int32_t*>(to_ptr(a[2], at::kInt, s.N_pad));
    auto* inv = static_cast<int32_t*>(to_ptr(a[3], at::kInt, s.N));
    auto* blk_valid = static_cast<int32_t*>(to_ptr(a[4], at::kInt, s.M));
    int64_t ws_bytes = 0;
    void* ws = to_ptr(a[5], at::ScalarType::Undefined, 0, &ws_bytes);
    void* st = stream();
    PyThreadState* gil = PyEval_SaveThread();
    const int rc = dfs_token_order(&g, order, perm_pad, inv, blk_valid, ws, size_t(ws_bytes), st);
    PyEval_RestoreThread(gil);
    return rc;
  });
}

// The staged calls.  Their arguments as binding.py passes them on, None where it takes None.
void* to_ptr_or_null(PyObject* x, at::ScalarType type, int64_t numel, int64_t* bytes = nullptr) {
  return x == Py_None ? nullptr : to_ptr(x, type, numel, bytes);
}
at::ScalarType tensor_type(int dtype) { return dtype == DFS_E4M3 ? at::kFloat8_e4m3fn : dtype == DFS_BF16 ? at::kBFloat16 : at::kFloat; }
struct Problem {
  dfs_geom g;
  dfs_sizes s;
  explicit Problem(PyObject* x) : g(to_geom(x)) { need(dfs_geom_sizes(&g, &s) == DFS_OK); }
  int64_t source() const { return int64_t(g.heads) * s.N * g.d; }
  int64_t ordered() const { return int64_t(g.heads) * s.N_pad * g.d; }
  int64_t scores() const { return int64_t(g.heads) * s.M_v * s.M_v; }
  int64_t rows() const { return int64_t(g.heads) * s.M; }
};
template <class F>
int without_gil(F f) {
  PyThreadState* gil = PyEval_SaveThread();
  const int rc = f();
  PyEval_RestoreThread(gil);
  return rc;
}

template <bool BACK>
PyObject* reorder(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 5);
    const Problem p(a[0]);
    const int dtype = to_int(a[1]);
    const auto type = tensor_type(dtype);
    const void* x = to_ptr(a[2], type, BACK ? p.ordered() : p.source());
    const auto* index = static_cast<const int32_t*>(to_ptr(a[3], at::kInt, BACK ? p.s.N : p.s.N_pad));
    void *y = to_ptr(a[4], type, BACK ? p.source() : p.ordered()), *st = stream();
    return without_gil([&] { return BACK ? dfs_unperm(&p.g, dtype, x, index, y, st) : dfs_permute(&p.g, dtype, x, index, y, st); });
  });
}

PyObject* block_score(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 6);
    const Problem p(a[0]);
    const int dtype = to_int(a[1]);
    const void *q = to_ptr(a[2], tensor_type(dtype), p.ordered()), *k = to_ptr(a[3], tensor_type(dtype), p.ordered());
    auto* score = static_cast<float*>(to_ptr(a[4], at::kFloat, p.scores()));
    int64_t ws_bytes = 0;
    void *ws = to_ptr(a[5], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    return without_gil([&] { return dfs_block_score(&p.g, dtype, q, k, score, ws, size_t(ws_bytes), st); });
  });
}

PyObject* select_mask(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 11);
    const Problem p(a[0]);
    const auto* score = static_cast<const float*>(to_ptr(a[1], at::kFloat, p.scores()));
    const int mode = to_int(a[2]), K_max = to_int(a[8]);
    const double sparsity = to_double(a[3]), mass = to_double(a[4]);
    auto* mask = static_cast<uint8_t*>(to_ptr_or_null(a[5], at::kByte, p.rows() * p.s.M));
    auto *kv_idx = static_cast<int32_t*>(to_ptr(a[6], at::kInt, p.rows() * K_max)), *kv_cnt = static_cast<int32_t*>(to_ptr(a[7], at::kInt, p.rows()));
    auto* k_head = static_cast<int32_t*>(to_ptr_or_null(a[9], at::kInt, p.g.heads));
    int64_t ws_bytes = 0;
    void *ws = to_ptr_or_null(a[10], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    return without_gil([&] { return dfs_select_mask(&p.g, score, mode, sparsity, mass, mask, kv_idx, kv_cnt, K_max, k_head, ws, size_t(ws_bytes), st); });
  });
}

PyObject* sparse_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 11);
    const Problem p(a[0]);
    const int dtype = to_int(a[1]), K_max = to_int(a[7]);
    const auto type = tensor_type(dtype);
    const void *q = to_ptr(a[2], type, p.ordered()), *k = to_ptr(a[3], type, p.ordered()), *v = to_ptr(a[4], type, p.ordered());
    const auto *kv_idx = static_cast<const int32_t*>(to_ptr(a[5], at::kInt, p.rows() * K_max)),
               *kv_cnt = static_cast<const int32_t*>(to_ptr(a[6], at::kInt, p.rows()));
    const float scale = float(to_double(a[8]));
    void* o = to_ptr(a[9], type, p.ordered());
    auto* lse = static_cast<float*>(to_ptr_or_null(a[10], at::kFloat, int64_t(p.g.heads) * p.s.N_pad));
    void* st = stream();
    return without_gil([&] { return dfs_sparse_attn_fwd(&p.g, dtype, q, k, v, kv_idx, kv_cnt, K_max, scale, o, lse, st); });
  });
}

PyObject* recall(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 4);
    const Problem p(a[0]);
    const int64_t rows = int64_t(p.g.heads) * p.s.N_pad;
    const auto *kept = static_cast<const float*>(to_ptr(a[1], at::kFloat, rows)), *all = static_cast<const float*>(to_ptr(a[2], at::kFloat, rows));
    auto* out = static_cast<float*>(to_ptr(a[3], at::kFloat, p.g.heads));
    void* st = stream();
    return without_gil([&] { return dfs_recall(&p.g, kept, all, out, st); });
  });
}

// Norm and rotation of queries and keys, and windowed attention.  As binding.py has them: tensors of given shapes on the current device, whose rows are
// dense, None where it takes None.
struct Here {
  int device;
  Here() : device(int(c10::hip::current_device())) {}

  const at::Tensor& tensor(PyObject* x, at::ScalarType type) const {
    need(THPVariable_CheckExact(x));
    const at::Tensor& t = THPVariable_Unpack(x);
    need(t.is_cuda() && t.get_device() == device && (type == at::ScalarType::Undefined || t.scalar_type() == type));
    return t;
  }
  struct MaybeView {
    dfs_view v;
    bool there;
    const dfs_view* get() const { return there ? &v : nullptr; }
  };
  MaybeView view(PyObject* x, int dtype, int64_t batch, int64_t heads, int64_t rows, int64_t d) const {
    MaybeView r = {};
    if (x == Py_None) return r;
    const at::Tensor& t = tensor(x, tensor_type(dtype));
    need(t.dim() == 4);
    const auto n = t.sizes(), s = t.strides();
    need(n[0] == batch && n[1] == heads && n[2] == rows && n[3] == d && (s[3] == 1 || t.numel() == 0));
    r.v = dfs_view{t.data_ptr(), s[0], s[1], s[2]};
    r.there = true;
    return r;
  }
  // Of one batch, without that axis.
  MaybeView flat_view(PyObject* x, int dtype, int64_t heads, int64_t rows, int64_t d) const {
    MaybeView r = {};
    if (x == Py_None) return r;
    const at::Tensor& t = tensor(x, tensor_type(dtype));
    need(t.dim() == 3);
    const auto n = t.sizes(), s = t.strides();
    need(n[0] == heads && n[1] == rows && n[2] == d && (s[2] == 1 || t.numel() == 0));
    r.v = dfs_view{t.data_ptr(), 0, s[0], s[1]};
    r.there = true;
    return r;
  }
  template <class T> T* flat(PyObject* x, at::ScalarType type, int64_t numel, int64_t* bytes = nullptr) const {
    if (x == Py_None) return nullptr;
    const at::Tensor& t = tensor(x, type);
    need(t.is_contiguous() && t.numel() >= numel);
    if (bytes) *bytes = t.numel() * int64_t(t.element_size());
    return static_cast<T*>(t.data_ptr());
  }
  const int32_t* positions(const dfs_qk_geom& g, PyObject* x, int64_t* pos_batch) const {
    const at::Tensor& t = tensor(x, at::kInt);
    const auto n = t.sizes();
    const int64_t dim = t.dim();
    need(t.is_contiguous() && (dim == 2 || (dim == 3 && (n[0] == 1 || n[0] == g.batch))) && n[dim - 2] == g.tokens && n[dim - 1] == g.axes);
    *pos_batch = dim == 3 && n[0] == g.batch && g.batch > 1 ? int64_t(g.tokens) * g.axes : 0;
    return static_cast<const int32_t*>(t.data_ptr());
  }
};

PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 12);
    const auto g = to_struct<dfs_qk_geom>(a[0], g_qk_type);
    const int dtype = to_int(a[1]);
    const Here here;
    const auto type = tensor_type(dtype);
    int64_t pos_batch = 0;
    const int32_t* pos = here.positions(g, a[5], &pos_batch);
    const auto* start = here.flat<const int32_t>(a[11], at::kInt, g.batch);
    int64_t rows = g.tokens;
    if (start) {
      const at::Tensor& cache = here.tensor(a[9], type);
      need(cache.dim() == 4);
      rows = cache.size(2);
      need(rows == int64_t(int32_t(rows)));
    }
    const auto q = here.view(a[2], dtype, g.batch, g.heads, g.tokens, g.d), k = here.view(a[3], dtype, g.batch, g.heads_kv, g.tokens, g.d),
               v = here.view(a[4], dtype, g.batch, g.heads_kv, g.tokens, g.d), q_out = here.view(a[8], dtype, g.batch, g.heads, g.tokens, g.d),
               k_out = here.view(a[9], dtype, g.batch, g.heads_kv, rows, g.d), v_out = here.view(a[10], dtype, g.batch, g.heads_kv, rows, g.d);
    const auto *w_q = here.flat<const float>(a[6], at::kFloat, g.d), *w_k = here.flat<const float>(a[7], at::kFloat, g.d);
    void* st = stream();
    return without_gil([&] {
      return dfs_qk_norm_rope(&g, dtype, q.get(), k.get(), v.get(), pos, pos_batch, w_q, w_k, q_out.get(), k_out.get(), v_out.get(), start, int32_t(rows), st);
    });
  });
}

PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 16);
    const auto g = to_struct<dfs_qk_geom>(a[0], g_qk_type);
    const int dtype = to_int(a[1]);
    const Here here;
    int64_t pos_batch = 0, ws_bytes = 0;
    const int32_t* pos = here.positions(g, a[4], &pos_batch);
    const auto heads = [&](PyObject* x) { return here.view(x, dtype, g.batch, g.heads, g.tokens, g.d); };
    const auto heads_kv = [&](PyObject* x) { return here.view(x, dtype, g.batch, g.heads_kv, g.tokens, g.d); };
    const auto q = heads(a[2]), k = heads_kv(a[3]), dq_out = heads(a[7]), dk_out = heads_kv(a[8]), dv_out = heads_kv(a[9]), dq = heads(a[10]),
               dk = heads_kv(a[11]), dv = heads_kv(a[12]);
    const auto *w_q = here.flat<const float>(a[5], at::kFloat, g.d), *w_k = here.flat<const float>(a[6], at::kFloat, g.d);
    auto *dw_q = here.flat<float>(a[13], at::kFloat, g.d), *dw_k = here.flat<float>(a[14], at::kFloat, g.d);
    void *ws = here.flat<void>(a[15], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    return without_gil([&] {
      return dfs_qk_norm_rope_bwd(&g, dtype, q.get(), k.get(), pos, pos_batch, w_q, w_k, dq_out.get(), dk_out.get(), dv_out.get(), dq.get(), dk.get(),
                                  dv.get(), dw_q, dw_k, ws, size_t(ws_bytes), st);
    });
  });
}

template <bool BACK>
PyObject* window_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == (BACK ? 15 : 11));
    const auto w = to_struct<dfs_window>(a[0], g_window_type);
    const int dtype = to_int(a[1]);
    const Here here;
    int64_t ws_bytes = 0;
    const auto of_q = [&](PyObject* x) { return here.view(x, dtype, w.batch, w.heads, w.n_q, w.d); };
    const auto of_k = [&](PyObject* x) { return here.view(x, dtype, w.batch, w.heads_kv, w.n_k, w.d); };
    const auto q = of_q(a[2]), k = of_k(a[3]), v = of_k(a[4]), o = of_q(a[BACK ? 5 : 8]);
    auto* lse = here.flat<float>(a[BACK ? 6 : 9], at::kFloat, int64_t(w.batch) * w.heads * w.n_q);
    PyObject* const* len = a + (BACK ? 8 : 5);
    const auto *q_len = here.flat<const int32_t>(len[0], at::kInt, w.batch), *k_len = here.flat<const int32_t>(len[1], at::kInt, w.batch);
    const float scale = float(to_double(len[2]));
    void *ws = here.flat<void>(a[n - 1], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    if (!BACK)
      return without_gil([&] { return dfs_window_attn_fwd(&w, dtype, q.get(), k.get(), v.get(), q_len, k_len, scale, o.get(), lse, ws, size_t(ws_bytes), st); });
    const auto d_o = of_q(a[7]), dq = of_q(a[BACK ? 11 : 0]), dk = of_k(a[BACK ? 12 : 0]), dv = of_k(a[BACK ? 13 : 0]);
    return without_gil([&] {
      return dfs_window_attn_bwd(&w, dtype, q.get(), k.get(), v.get(), o.get(), lse, d_o.get(), q_len, k_len, scale, dq.get(), dk.get(), dv.get(), ws,
                                 size_t(ws_bytes), st);
    });
  });
}

template <bool BACK>
PyObject* packed_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == (BACK ? 15 : 11));
    const auto w = to_struct<dfs_packed>(a[0], g_packed_type);
    const int dtype = to_int(a[1]);
    const Here here;
    int64_t ws_bytes = 0;
    const auto of_q = [&](PyObject* x) { return here.flat_view(x, dtype, w.heads, w.n_q, w.d); };
    const auto of_k = [&](PyObject* x) { return here.flat_view(x, dtype, w.heads_kv, w.n_k, w.d); };
    const auto q = of_q(a[2]), k = of_k(a[3]), v = of_k(a[4]), o = of_q(a[BACK ? 5 : 8]);
    auto* lse = here.flat<float>(a[BACK ? 6 : 9], at::kFloat, int64_t(w.heads) * w.n_q);
    PyObject* const* start = a + (BACK ? 8 : 5);
    const auto *q_start = here.flat<const int32_t>(start[0], at::kInt, int64_t(w.seqs) + 1), *k_start = here.flat<const int32_t>(start[1], at::kInt, int64_t(w.seqs) + 1);
    const float scale = float(to_double(start[2]));
    void *ws = here.flat<void>(a[n - 1], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    if (!BACK)
      return without_gil([&] { return dfs_packed_attn_fwd(&w, dtype, q.get(), k.get(), v.get(), q_start, k_start, scale, o.get(), lse, ws, size_t(ws_bytes), st); });
    const auto d_o = of_q(a[7]), dq = of_q(a[BACK ? 11 : 0]), dk = of_k(a[BACK ? 12 : 0]), dv = of_k(a[BACK ? 13 : 0]);
    return without_gil([&] {
      return dfs_packed_attn_bwd(&w, dtype, q.get(), k.get(), v.get(), o.get(), lse, d_o.get(), q_start, k_start, scale, dq.get(), dk.get(), dv.get(), ws,
                                 size_t(ws_bytes), st);
    });
  });
}

// binding.Pages; its tensors are held while the call runs.
struct PagesOf {
  const Attr k, v, table, k_scale, v_scale;
  dfs_pages p = {};
  PagesOf(const Here& here, PyObject* x, int64_t seqs, int64_t heads_kv, int64_t d)
      : k(x, s_k), v(x, s_v), table(x, s_table), k_scale(x, s_k_scale), v_scale(x, s_v_scale) {
    const at::Tensor &t = here.tensor(k.o, at::ScalarType::Undefined), &rows = here.tensor(table.o, at::kInt);
    p.dtype = t.scalar_type() == at::kFloat ? DFS_F32 : t.scalar_type() == at::kBFloat16 ? DFS_BF16 : DFS_E4M3;
    need(t.scalar_type() == tensor_type(p.dtype) && t.dim() == 4 && rows.dim() == 2 && rows.size(0) == seqs && rows.is_contiguous());
    const int64_t n = t.size(0), page = t.size(2), row = rows.size(1);
    need(n == int64_t(int32_t(n)) && page == int64_t(int32_t(page)) && row == int64_t(int32_t(row)));
    p.pages = int32_t(n);
    p.page = int32_t(page);
    p.table_row = int32_t(row);
    p.k = here.view(k.o, p.dtype, n, heads_kv, page, d).v;
    const auto values = here.view(v.o, p.dtype, n, heads_kv, page, d);
    need(values.there);
    p.v = values.v;
    p.table = static_cast<const int32_t*>(rows.data_ptr());
    p.k_scale = here.flat<float>(k_scale.o, at::kFloat, n * heads_kv);
    p.v_scale = here.flat<float>(v_scale.o, at::kFloat, n * heads_kv);
  }
};

PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 13);
    const auto g = to_struct<dfs_qk_geom>(a[0], g_qk_type);
    const int dtype = to_int(a[1]), norm = PyObject_IsTrue(a[12]);
    need(norm >= 0);
    const Here here;
    const auto rows = [&](PyObject* x, int64_t heads) { return here.flat_view(x, dtype, heads, g.tokens, g.d); };
    const auto q = rows(a[2], g.heads), k = rows(a[3], g.heads_kv), v = rows(a[4], g.heads_kv), q_out = rows(a[10], g.heads);
    const auto *q_start = here.flat<const int32_t>(a[5], at::kInt, int64_t(g.batch) + 1), *k_len = here.flat<const int32_t>(a[6], at::kInt, g.batch);
    const int32_t* pos = nullptr;
    if (a[7] != Py_None) {
      const at::Tensor& t = here.tensor(a[7], at::kInt);
      need(t.is_contiguous() && t.dim() == 2 && t.size(0) == g.tokens && t.size(1) == g.axes);
      pos = static_cast<const int32_t*>(t.data_ptr());
    }
    const auto *w_q = here.flat<const float>(a[8], at::kFloat, g.d), *w_k = here.flat<const float>(a[9], at::kFloat, g.d);
    const PagesOf pages(here, a[11], g.batch, g.heads_kv, g.d);
    void* st = stream();
    return without_gil([&] {
      return dfs_paged_append(&g, dtype, q.get(), k.get(), v.get(), q_start, k_len, pos, w_q, w_k, q_out.get(), &pages.p, norm, st);
    });
  });
}

PyObject* paged_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    need(n == 10);
    const auto w = to_struct<dfs_paged>(a[0], g_paged_type);
    const int dtype = to_int(a[1]);
    const Here here;
    int64_t ws_bytes = 0;
    const auto q = here.flat_view(a[2], dtype, w.heads, w.n_q, w.d), o = here.flat_view(a[7], dtype, w.heads, w.n_q, w.d);
    const PagesOf pages(here, a[3], w.seqs, w.heads_kv, w.d);
    const auto *q_start = here.flat<const int32_t>(a[4], at::kInt, int64_t(w.seqs) + 1), *k_len = here.flat<const int32_t>(a[5], at::kInt, w.seqs);
    const float scale = float(to_double(a[6]));
    auto* lse = here.flat<float>(a[8], at::kFloat, int64_t(w.heads) * w.n_q);
    void *ws = here.flat<void>(a[9], at::ScalarType::Undefined, 0, &ws_bytes), *st = stream();
    return without_gil([&] { return dfs_paged_attn_fwd(&w, dtype, q.get(), &pages.p, q_start, k_len, scale, o.get(), lse, ws, size_t(ws_bytes), st); });
  });
}

PyObject* set_layer_types(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n == 4) {
    for (int i = 0; i < 4; ++i) Py_INCREF(a[i]);
    g_qk_type = a[0];
    g_window_type = a[1];
    g_packed_type = a[2];
    g_paged_type = a[3];
  }
  Py_RETURN_NONE;
}

PyObject* set_geom_type(PyObject*, PyObject* type) {
  Py_INCREF(type);
  g_geom_type = type;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(forward)), METH_FASTCALL, nullptr},
    {"token_order", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(token_order)), METH_FASTCALL, nullptr},
    {"permute", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(reorder<false>)), METH_FASTCALL, nullptr},
    {"unperm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(reorder<true>)), METH_FASTCALL, nullptr},
    {"block_score", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_score)), METH_FASTCALL, nullptr},
    {"select_mask", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(select_mask)), METH_FASTCALL, nullptr},
    {"sparse_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sparse_attn)), METH_FASTCALL, nullptr},
    {"recall", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(recall)), METH_FASTCALL, nullptr},
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm_rope)), METH_FASTCALL, nullptr},
    {"qk_norm_rope_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm_rope_bwd)), METH_FASTCALL, nullptr},
    {"window_attn_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(window_attn<false>)), METH_FASTCALL, nullptr},
    {"window_attn_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(window_attn<true>)), METH_FASTCALL, nullptr},
    {"packed_attn_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(packed_attn<false>)), METH_FASTCALL, nullptr},
    {"packed_attn_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(packed_attn<true>)), METH_FASTCALL, nullptr},
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, nullptr},
    {"paged_attn_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attn)), METH_FASTCALL, nullptr},
    {"set_geom_type", set_geom_type, METH_O, nullptr},
    {"set_layer_types", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(set_layer_types)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  s_kv_idx = PyUnicode_InternFromString("kv_idx");
  s_kv_cnt = PyUnicode_InternFromString("kv_cnt");
  s_mask = PyUnicode_InternFromString("mask");
  s_k_head = PyUnicode_InternFromString("k_head");
  s_K_max = PyUnicode_InternFromString("K_max");
  s_k = PyUnicode_InternFromString("k");
  s_v = PyUnicode_InternFromString("v");
  s_table = PyUnicode_InternFromString("table");
  s_k_scale = PyUnicode_InternFromString("k_scale");
  s_v_scale = PyUnicode_InternFromString("v_scale");
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", DFS_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
