// Python entry points of the hot-path calls: argument checks, output allocation, workspace lookup and
// the C-ABI call in one native function each.  The same work in Python (ctypes marshalling of twenty
// arguments, torch.empty, the stream lookup) and the C call took 24 us a call on the host, longer than
// the kernels of a small call; both take 8 us now (a decode step of one sequence: 24.7 -> 10.7 us a
// step, a turn of one request, two calls: 54 -> 39 us).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "recache.h"

namespace {

// The library's functions, by the addresses that the binding resolved when it loaded it.
struct Lib {
  decltype(&recache_encode_workspace_bytes) encode_ws;
  decltype(&recache_compact_workspace_bytes) compact_ws;
  decltype(&recache_prefill_workspace_bytes) prefill_ws;
  decltype(&recache_prefill_history_workspace_bytes) prefill_history_ws;
  decltype(&recache_decode_workspace_bytes) decode_ws;
  decltype(&recache_encode_resources) encode;
  decltype(&recache_compact_routes) compact;
  decltype(&recache_attend_prefill) prefill;
  decltype(&recache_attend_prefill_gather) prefill_gather;
  decltype(&recache_attend_prefill_history) prefill_history;
  decltype(&recache_attend_decode) decode;
  decltype(&recache_attend_decode_gather) decode_gather;
  decltype(&recache_compact_routes_q8) compact_q8;
  decltype(&recache_decode_q8_workspace_bytes) decode_q8_ws;
  decltype(&recache_decode_weighted_workspace_bytes) decode_weighted_ws;
  decltype(&recache_attend_decode_q8) decode_q8;
  decltype(&recache_attend_decode_weighted) decode_weighted;
  decltype(&recache_evict_rows) evict;
} lib;

PyObject *s_ws, *s_workspace, *s_check, *s_shape;   // interned attribute names of the Python context object

struct Error {};   // a Python exception has been set

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "expected a tensor"); throw Error(); }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || !t.is_contiguous()) { PyErr_SetString(PyExc_AssertionError, "device, contiguous tensors only"); throw Error(); }
  return t;
}
void* ptr(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
template <typename T> T* ptr_as(PyObject* o) { return static_cast<T*>(ptr(o)); }
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {   // numpy integers and the like
    PyErr_Clear();
    PyObject* i = PyNumber_Long(o);
    if (!i) throw Error();
    const long long w = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (w == -1 && PyErr_Occurred()) throw Error();
    return w;
  }
  return v;
}

// What every call carries: the context object, its handle and its storage dtype.
struct Ctx {
  PyObject* self; recache_ctx* h; int dtype;
  explicit Ctx(PyObject* const* a) : self(a[0]), h(nullptr), dtype((int)integer(a[2])) {
    if (a[1] != Py_None) h = static_cast<recache_ctx*>(PyLong_AsVoidPtr(a[1]));
    if (PyErr_Occurred()) throw Error();
  }
  // the caller's workspace, or the context's own, grown by its Python method
  at::Tensor workspace(PyObject* given, int64_t need) const {
    if (given != Py_None) return tensor(given);
    PyObject* ws = PyObject_GetAttr(self, s_ws);
    if (!ws) throw Error();
    if (ws == Py_None || !THPVariable_Check(ws) || THPVariable_Unpack(ws).numel() < (need > 256 ? need : 256)) {
      Py_DECREF(ws);
      PyObject* n = PyLong_FromLongLong(need);
      ws = PyObject_CallMethodObjArgs(self, s_workspace, n, nullptr);
      Py_XDECREF(n);
      if (!ws) throw Error();
    }
    at::Tensor t = THPVariable_Unpack(ws);
    Py_DECREF(ws);
    return t;
  }
  at::ScalarType out_type(PyObject* out_dtype) const {
    if (out_dtype == Py_None) return dtype == RECACHE_F32 ? at::kFloat : at::kBFloat16;
    if (!THPDtype_Check(out_dtype)) { PyErr_SetString(PyExc_TypeError, "out_dtype must be a torch.dtype"); throw Error(); }
    return reinterpret_cast<THPDtype*>(out_dtype)->scalar_type;
  }
  void check(recache_status st, const char* what) const {
    if (st == RECACHE_OK) return;
    PyObject* n = PyLong_FromLong(st);
    PyObject* w = PyUnicode_FromString(what);
    PyObject* r = PyObject_CallMethodObjArgs(self, s_check, n, w, nullptr);   // raises
    Py_XDECREF(n); Py_XDECREF(w); Py_XDECREF(r);
    throw Error();
  }
};
int out_code(at::ScalarType t) { return t == at::kFloat ? RECACHE_F32 : RECACHE_BF16; }
at::Tensor given_or_empty(PyObject* o, at::IntArrayRef sizes, at::ScalarType t, const at::Tensor& like) {
  if (o != Py_None) return tensor(o);
  return at::empty(sizes, at::TensorOptions().dtype(t).device(like.device()));
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Other Python threads run while the launches are made.  (The lock is taken again also where f throws: a tensor
// without memory does when it is asked for its address.)
struct Unlock {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlock() { PyEval_RestoreThread(state); }
};
template <typename F> recache_status unlocked(F f) {
  const Unlock u;
  return f();
}

// Runs a call's body; exceptions become Python ones.
template <typename F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n); return nullptr; }
  try {
    return f();
  } catch (const Error&) {
    return nullptr;
  } catch (const std::exception&) {
    torch::translate_exception_to_python(std::current_exception());   // OutOfMemoryError, IndexError ... as torch raises them
    return nullptr;
  }
}

PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n) {   // ctx x3, q k v cu max_len slot k_cache v_cache out out_dtype workspace
  return guarded(n, 14, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &q = tensor(a[3]), &cu = tensor(a[6]), &kc = tensor(a[9]);
    const at::ScalarType ot = c.out_type(a[12]);
    const at::Tensor out = given_or_empty(a[11], q.sizes(), ot, q);
    const int n_res = (int)cu.numel() - 1, total = (int)q.size(0), max_len = (int)integer(a[7]);
    const at::Tensor ws = c.workspace(a[13], lib.encode_ws(c.h, n_res, total, max_len));
    void *k = ptr(a[4]), *v = ptr(a[5]), *vc = ptr(a[10]);
    const int32_t* slot = ptr_as<int32_t>(a[8]);
    c.check(unlocked([&] {
      return lib.encode(c.h, q.data_ptr(), k, v, (const int32_t*)cu.data_ptr(), n_res, total, max_len, slot, kc.data_ptr(), vc, kc.size(1),
                        out.data_ptr(), out_code(ot), ws.data_ptr(), ws.numel(), stream());
    }), "recache_encode_resources");
    return THPVariable_Wrap(out);
  });
}

// ctx x3, k_cache v_cache keep res_off res_slot res_len vis mode route_cu route_idx k_out v_out route_len page_table free_pages workspace
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &kc = tensor(a[3]), &res_off = tensor(a[6]), &res_slot = tensor(a[7]), &route_idx = tensor(a[12]);
    const int n_req = (int)res_off.numel() - 1, listed = (int)res_slot.numel(), mode = (int)integer(a[10]);
    const bool paged = mode == RECACHE_PAGED;
    const at::Tensor ws = c.workspace(a[18], lib.compact_ws(c.h, n_req, listed));
    int64_t capacity = route_idx.numel(), n_free = 0, n_pool = 0;
    int max_pages = 0;
    if (paged) {
      max_pages = (int)tensor(a[16]).size(1); n_free = tensor(a[17]).numel(); n_pool = tensor(a[13]).size(0);
    } else if (a[13] != Py_None) {
      capacity = std::min(capacity, tensor(a[13]).size(0));
    }
    void *vc = ptr(a[4]), *k_out = ptr(a[13]), *v_out = ptr(a[14]);
    const uint8_t *keep = ptr_as<uint8_t>(a[5]), *vis = ptr_as<uint8_t>(a[9]);
    int32_t *res_len = ptr_as<int32_t>(a[8]), *route_cu = ptr_as<int32_t>(a[11]), *route_len = ptr_as<int32_t>(a[15]),
            *table = ptr_as<int32_t>(a[16]), *free_pages = ptr_as<int32_t>(a[17]);
    c.check(unlocked([&] {
      return lib.compact(c.h, kc.data_ptr(), vc, kc.size(1), keep, (const int32_t*)res_off.data_ptr(), (const int32_t*)res_slot.data_ptr(),
                         res_len, n_req, listed, vis, mode, route_cu, route_len, (int32_t*)route_idx.data_ptr(), capacity, k_out, v_out, table,
                         max_pages, free_pages, n_free, n_pool, ws.data_ptr(), ws.numel(), stream());
    }), "recache_compact_routes");
    Py_RETURN_NONE;
  });
}

// ctx x3, q k v cu_q q_pos0 max_q k_route v_route route_cu k_conv_out v_conv_out out out_dtype workspace [route_idx: gather, k/v_route = caches]
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 18, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &q = tensor(a[3]), &k = tensor(a[4]), &cu = tensor(a[6]), &kr = tensor(a[9]);
    const int n_req = (int)cu.numel() - 1, total = (int)q.size(0), max_q = (int)integer(a[8]);
    const at::ScalarType ot = c.out_type(a[15]);
    const at::Tensor out = given_or_empty(a[14], q.sizes(), ot, q);
    const std::array<int64_t, 3> conv = {k.size(1), total, k.size(2)};
    const at::Tensor ko = given_or_empty(a[12], conv, k.scalar_type(), q), vo = given_or_empty(a[13], conv, k.scalar_type(), q);
    const at::Tensor ws = c.workspace(a[16], lib.prefill_ws(c.h, n_req, total, max_q));
    void *v = ptr(a[5]), *vr = ptr(a[10]);
    const int32_t *pos0 = ptr_as<int32_t>(a[7]), *route_cu = ptr_as<int32_t>(a[11]);
    if (a[17] == Py_None) {
      c.check(unlocked([&] {
        return lib.prefill(c.h, q.data_ptr(), k.data_ptr(), v, (const int32_t*)cu.data_ptr(), pos0, n_req, total, max_q, kr.data_ptr(), vr, route_cu,
                           kr.size(0), ko.data_ptr(), vo.data_ptr(), out.data_ptr(), out_code(ot), ws.data_ptr(), ws.numel(), stream());
      }), "recache_attend_prefill");
    } else {
      const at::Tensor& idx = tensor(a[17]);
      c.check(unlocked([&] {
        return lib.prefill_gather(c.h, q.data_ptr(), k.data_ptr(), v, (const int32_t*)cu.data_ptr(), pos0, n_req, total, max_q, kr.data_ptr(), vr,
                                  kr.size(1), (const int32_t*)idx.data_ptr(), route_cu, idx.numel(), ko.data_ptr(), vo.data_ptr(), out.data_ptr(),
                                  out_code(ot), ws.data_ptr(), ws.numel(), stream());
      }), "recache_attend_prefill_gather");
    }
    PyObject* r = PyTuple_New(3);
    if (!r) throw Error();
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(ko));
    PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(vo));
    return r;
  });
}

// ctx x3, q k v cu_q q_pos0 max_q k_route v_route route_cu k_cache v_cache conv_slot hist_len out out_dtype workspace
PyObject* prefill_history(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &q = tensor(a[3]), &cu = tensor(a[6]), &kr = tensor(a[9]), &kc = tensor(a[12]);
    const int n_req = (int)cu.numel() - 1, total = (int)q.size(0), max_q = (int)integer(a[8]);
    const at::ScalarType ot = c.out_type(a[17]);
    const at::Tensor out = given_or_empty(a[16], q.sizes(), ot, q);
    const at::Tensor ws = c.workspace(a[18], lib.prefill_history_ws(c.h, n_req, total, max_q));
    void *k = ptr(a[4]), *v = ptr(a[5]), *vr = ptr(a[10]), *vc = ptr(a[13]);
    const int32_t *pos0 = ptr_as<int32_t>(a[7]), *route_cu = ptr_as<int32_t>(a[11]), *slot = ptr_as<int32_t>(a[14]), *hist = ptr_as<int32_t>(a[15]);
    c.check(unlocked([&] {
      return lib.prefill_history(c.h, q.data_ptr(), k, v, (const int32_t*)cu.data_ptr(), pos0, n_req, total, max_q, kr.data_ptr(), vr, route_cu,
                                 kr.size(0), kc.data_ptr(), vc, kc.size(1), slot, hist, out.data_ptr(), out_code(ot), ws.data_ptr(), ws.numel(),
                                 stream());
    }), "recache_attend_prefill_history");
    return THPVariable_Wrap(out);
  });
}

// ctx x3, q q_pos k_pages v_pages res_table res_len hist_table hist_len k_new v_new out out_dtype workspace
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &q = tensor(a[3]), &kp = tensor(a[5]), &rt = tensor(a[7]), &ht = tensor(a[9]);
    const int batch = (int)q.size(0), mr = (int)rt.size(1), mh = (int)ht.size(1);
    const at::ScalarType ot = c.out_type(a[14]);
    const at::Tensor out = given_or_empty(a[13], q.sizes(), ot, q);
    const at::Tensor ws = c.workspace(a[15], lib.decode_ws(c.h, batch, mr, mh));
    void *vp = ptr(a[6]), *kn = ptr(a[11]), *vn = ptr(a[12]);
    const int32_t *pos = ptr_as<int32_t>(a[4]), *rl = ptr_as<int32_t>(a[8]), *hl = ptr_as<int32_t>(a[10]);
    c.check(unlocked([&] {
      return lib.decode(c.h, q.data_ptr(), pos, batch, kn, vn, kp.data_ptr(), vp, kp.size(0), (const int32_t*)rt.data_ptr(), mr, rl,
                        (const int32_t*)ht.data_ptr(), mh, hl, out.data_ptr(), out_code(ot), ws.data_ptr(), ws.numel(), stream());
    }), "recache_attend_decode");
    return THPVariable_Wrap(out);
  });
}

// ctx x3, q q_pos k_cache v_cache route_idx route_cu max_res_pages k_pages v_pages hist_table hist_len k_new v_new out out_dtype workspace
PyObject* decode_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &q = tensor(a[3]), &kc = tensor(a[5]), &idx = tensor(a[7]), &kp = tensor(a[10]), &ht = tensor(a[12]);
    const int batch = (int)q.size(0), mr = (int)integer(a[9]), mh = (int)ht.size(1);
    const at::ScalarType ot = c.out_type(a[17]);
    const at::Tensor out = given_or_empty(a[16], q.sizes(), ot, q);
    const at::Tensor ws = c.workspace(a[18], lib.decode_ws(c.h, batch, mr, mh));
    void *vc = ptr(a[6]), *vp = ptr(a[11]), *kn = ptr(a[14]), *vn = ptr(a[15]);
    const int32_t *pos = ptr_as<int32_t>(a[4]), *cu = ptr_as<int32_t>(a[8]), *hl = ptr_as<int32_t>(a[13]);
    c.check(unlocked([&] {
      return lib.decode_gather(c.h, q.data_ptr(), pos, batch, kn, vn, kc.data_ptr(), vc, kc.size(1), (const int32_t*)idx.data_ptr(), cu, idx.numel(),
                               mr, kp.data_ptr(), vp, kp.size(0), (const int32_t*)ht.data_ptr(), mh, hl, out.data_ptr(), out_code(ot),
                               ws.data_ptr(), ws.numel(), stream());
    }), "recache_attend_decode_gather");
    return THPVariable_Wrap(out);
  });
}

// ---- 8-bit pages, weights and eviction: tensors of other types than the storage type meet in one call, so types and sizes are checked ----
[[noreturn]] void refuse(const char* what) { PyErr_SetString(PyExc_ValueError, what); throw Error(); }
const at::Tensor& typed(PyObject* o, at::ScalarType want, const char* what) {
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != want) refuse(what);
  return t;
}
const at::Tensor& i32(PyObject* o) { return typed(o, at::kInt, "lengths, positions and tables are int32"); }
const at::Tensor& f32(PyObject* o) { return typed(o, at::kFloat, "weights and scales are float32"); }
const at::Tensor& pages8(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kFloat8_e4m3fn && t.scalar_type() != at::kByte) refuse("8-bit pages are float8_e4m3fn or uint8");
  if (t.dim() != 3) refuse("pages are [n_pages][page_tokens][head_dim]");
  return t;
}
const at::Tensor& stored(const Ctx& c, PyObject* o) {
  return typed(o, c.dtype == RECACHE_F32 ? at::kFloat : at::kBFloat16, "queries, keys and values have the context's dtype");
}
const at::Tensor& pool(const Ctx& c, PyObject* o) {
  const at::Tensor& t = stored(c, o);
  if (t.dim() != 3) refuse("pages are [n_pages][page_tokens][head_dim]");
  return t;
}
const at::Tensor& table2(PyObject* o, int64_t rows) {
  const at::Tensor& t = i32(o);
  if (t.dim() != 2 || t.size(0) != rows) refuse("page tables are [items][pages]");
  return t;
}
void same(bool ok, const char* what) { if (!ok) refuse(what); }
// The context's sizes, and its device: the stream of a call is the one current there, whatever the current device is.
struct Sizes {
  int64_t v[5];
  explicit Sizes(const Ctx& c) {
    PyObject* t = PyObject_GetAttr(c.self, s_shape);
    if (!t) throw Error();
    for (int i = 0; i < 5; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
    Py_DECREF(t);
    if (PyErr_Occurred()) throw Error();
  }
  int64_t hq() const { return v[0]; }
  int64_t g() const { return v[1]; }
  int64_t d() const { return v[2]; }
  int64_t page_tokens() const { return v[3]; }
  // a pool of pages of the context's shape
  void pages(const at::Tensor& t) const {
    if (t.size(1) != page_tokens() || t.size(2) != d()) refuse("pages are [n_pages][page_tokens][head_dim] of the context");
  }
  template <typename... T> void here(const T&... t) const {
    if (((t.device().index() != v[4]) || ...)) refuse("tensors are on another device than the context");
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)v[4]).stream(); }
};

// ctx x3, k_cache v_cache keep res_off res_slot res_len vis route_cu route_idx k_pages8 v_pages8 k_scale v_scale page_table free_pages route_len
// workspace
PyObject* compact_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 20, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &kc = pool(c, a[3]), &vc = pool(c, a[4]), &res_off = i32(a[6]), &res_slot = i32(a[7]), &res_len = i32(a[8]), &cu = i32(a[10]),
                     &idx = i32(a[11]), &k8 = pages8(a[12]), &v8 = pages8(a[13]), &ks = f32(a[14]), &vs = f32(a[15]), &free_pages = i32(a[17]);
    const at::Tensor &keep = tensor(a[5]), &vis = tensor(a[9]);
    same(keep.element_size() == 1 && vis.element_size() == 1, "masks are uint8");
    const int64_t g = kc.size(0), n_req = res_off.numel() - 1, listed = res_slot.numel();
    const at::Tensor& table = table2(a[16], n_req * g);
    const Sizes sz(c);
    same(g == sz.g() && kc.size(2) == sz.d(), "caches are [KV heads][rows][head_dim] of the context");
    sz.pages(k8);
    sz.here(kc, vc, res_off, res_slot, res_len, cu, idx, k8, v8, ks, vs, free_pages, keep, vis, table);
    same(kc.sizes() == vc.sizes() && keep.numel() >= kc.size(1), "caches and keep mask differ in size");
    same(n_req >= 0 && res_len.numel() == listed && vis.numel() == g * listed && cu.numel() >= n_req * g + 1, "request lists differ in size");
    same(k8.sizes() == v8.sizes() && ks.numel() == k8.size(0) && vs.numel() == k8.size(0), "8-bit pages and scales differ in size");
    int32_t* lens = nullptr;
    if (a[18] != Py_None) {
      same(i32(a[18]).numel() >= n_req * g, "route_len is too short");
      sz.here(i32(a[18]));
      lens = ptr_as<int32_t>(a[18]);
    }
    const at::Tensor ws = c.workspace(a[19], lib.compact_ws(c.h, (int)n_req, (int)listed));
    sz.here(ws);
    c.check(unlocked([&] {
      return lib.compact_q8(c.h, kc.data_ptr(), vc.data_ptr(), kc.size(1), (const uint8_t*)keep.data_ptr(), (const int32_t*)res_off.data_ptr(),
                            (const int32_t*)res_slot.data_ptr(), (const int32_t*)res_len.data_ptr(), (int)n_req, (int)listed, (const uint8_t*)vis.data_ptr(),
                            (int32_t*)cu.data_ptr(), lens, (int32_t*)idx.data_ptr(), idx.numel(), (uint8_t*)k8.data_ptr(), (uint8_t*)v8.data_ptr(),
                            (float*)ks.data_ptr(), (float*)vs.data_ptr(), (int32_t*)table.data_ptr(), (int)table.size(1),
                            (const int32_t*)free_pages.data_ptr(), free_pages.numel(), k8.size(0), ws.data_ptr(), ws.nbytes(), sz.stream());
    }), "recache_compact_routes_q8");
    Py_RETURN_NONE;
  });
}

// What the two decode calls share: q, positions, pools, tables and the appended token.
struct DecodeIn {
  Sizes sz;
  const at::Tensor &q, &pos, &kp, &vp, &rl, &hl, &rt, &ht;
  const void *k_new, *v_new;
  const float* w_in; float* w_out;
  at::ScalarType ot; at::Tensor out;
  DecodeIn(const Ctx& c, PyObject* q_, PyObject* pos_, PyObject* kp_, PyObject* vp_, PyObject* rt_, PyObject* rl_, PyObject* ht_, PyObject* hl_, PyObject* kn,
           PyObject* vn, PyObject* wi, PyObject* wo, PyObject* out_, PyObject* out_dtype)
      : sz(c), q(stored(c, q_)), pos(i32(pos_)), kp(pool(c, kp_)), vp(pool(c, vp_)), rl(i32(rl_)), hl(i32(hl_)), rt(table2(rt_, rl.numel())),
        ht(table2(ht_, rl.numel())), k_new(nullptr), v_new(nullptr), w_in(nullptr), w_out(nullptr) {
    same(q.dim() == 3 && q.size(1) == sz.hq() && q.size(2) == sz.d() && pos.numel() == q.size(0),
         "q is [batch][query heads][head_dim] of the context, with a position for each sequence");
    same(rl.numel() == q.size(0) * sz.g() && hl.numel() == rl.numel(), "lengths are [batch x KV heads]");
    same(kp.sizes() == vp.sizes(), "pages differ in size");
    sz.pages(kp);
    sz.here(q, pos, kp, vp, rt, rl, ht, hl);
    same((kn == Py_None) == (vn == Py_None), "k_new and v_new go together");
    if (kn != Py_None) {
      const at::Tensor &k = stored(c, kn), &v = stored(c, vn);
      same(k.numel() == rl.numel() * q.size(2) && v.numel() == k.numel(), "k_new and v_new are [batch][KV heads][head_dim]");
      sz.here(k, v);
      k_new = k.data_ptr(); v_new = v.data_ptr();
    }
    const int64_t rows = kp.size(0) * kp.size(1);
    if (wi != Py_None) { sz.here(f32(wi)); same(f32(wi).numel() == rows, "weights are [n_pages][page_tokens]"); w_in = ptr_as<float>(wi); }
    if (wo != Py_None) { sz.here(f32(wo)); same(f32(wo).numel() == rows, "weights are [n_pages][page_tokens]"); w_out = ptr_as<float>(wo); }
    ot = out_ != Py_None ? tensor(out_).scalar_type() : c.out_type(out_dtype);
    same(ot == at::kFloat || ot == q.scalar_type(), "outputs are float32 or of the context's dtype");
    out = given_or_empty(out_, q.sizes(), ot, q);
    sz.here(out);
    same(out.numel() == q.numel(), "out has another size than q");
  }
};

// ctx x3, q q_pos k_pages8 v_pages8 k_scale v_scale res_table res_len k_pages v_pages hist_table hist_len k_new v_new weight_in weight_out out
// out_dtype workspace
PyObject* decode_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 22, [&]() -> PyObject* {
    const Ctx c(a);
    const DecodeIn d(c, a[3], a[4], a[11], a[12], a[9], a[10], a[13], a[14], a[15], a[16], a[17], a[18], a[19], a[20]);
    const at::Tensor &k8 = pages8(a[5]), &v8 = pages8(a[6]), &ks = f32(a[7]), &vs = f32(a[8]);
    d.sz.pages(k8);
    d.sz.here(k8, v8, ks, vs);
    same(k8.sizes() == v8.sizes() && ks.numel() == k8.size(0) && vs.numel() == k8.size(0), "8-bit pages and scales differ in size");
    const int batch = (int)d.q.size(0);
    const at::Tensor ws = c.workspace(a[21], d.w_out ? lib.decode_weighted_ws(c.h, batch, d.kp.size(0)) : lib.decode_q8_ws(c.h, batch));
    d.sz.here(ws);
    c.check(unlocked([&] {
      return lib.decode_q8(c.h, d.q.data_ptr(), (const int32_t*)d.pos.data_ptr(), batch, d.k_new, d.v_new, (const uint8_t*)k8.data_ptr(),
                           (const uint8_t*)v8.data_ptr(), (const float*)ks.data_ptr(), (const float*)vs.data_ptr(), k8.size(0), (const int32_t*)d.rt.data_ptr(),
                           (int)d.rt.size(1), (const int32_t*)d.rl.data_ptr(), d.kp.data_ptr(), d.vp.data_ptr(), d.kp.size(0), (const int32_t*)d.ht.data_ptr(),
                           (int)d.ht.size(1), (const int32_t*)d.hl.data_ptr(), d.w_in, d.w_out, d.out.data_ptr(), out_code(d.ot), ws.data_ptr(), ws.nbytes(),
                           d.sz.stream());
    }), "recache_attend_decode_q8");
    return THPVariable_Wrap(d.out);
  });
}

// ctx x3, q q_pos k_pages v_pages res_table res_len hist_table hist_len weight_out weight_in k_new v_new out out_dtype workspace
PyObject* decode_weighted(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 18, [&]() -> PyObject* {
    const Ctx c(a);
    const DecodeIn d(c, a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[13], a[14], a[12], a[11], a[15], a[16]);
    const int batch = (int)d.q.size(0);
    const at::Tensor ws = c.workspace(a[17], lib.decode_weighted_ws(c.h, batch, d.kp.size(0)));
    d.sz.here(ws);
    c.check(unlocked([&] {
      return lib.decode_weighted(c.h, d.q.data_ptr(), (const int32_t*)d.pos.data_ptr(), batch, d.k_new, d.v_new, d.kp.data_ptr(), d.vp.data_ptr(), d.kp.size(0),
                                 (const int32_t*)d.rt.data_ptr(), (int)d.rt.size(1), (const int32_t*)d.rl.data_ptr(), (const int32_t*)d.ht.data_ptr(),
                                 (int)d.ht.size(1), (const int32_t*)d.hl.data_ptr(), d.w_in, d.w_out, d.out.data_ptr(), out_code(d.ot), ws.data_ptr(),
                                 ws.nbytes(), d.sz.stream());
    }), "recache_attend_decode_weighted");
    return THPVariable_Wrap(d.out);
  });
}

// ctx x3, k_pages v_pages weight table row_len budget n_recent free_pages new_table new_len kept
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const Ctx c(a);
    const at::Tensor &kp = pool(c, a[3]), &vp = pool(c, a[4]), &w = f32(a[5]), &len = i32(a[7]), &table = table2(a[6], len.numel()), &free_pages = i32(a[10]),
                     &new_table = table2(a[11], len.numel()), &new_len = i32(a[12]), &kept = i32(a[13]);
    const long long budget = integer(a[8]), recent = integer(a[9]);
    const Sizes sz(c);
    sz.pages(kp);
    sz.here(kp, vp, w, len, table, free_pages, new_table, new_len, kept);
    same(kp.sizes() == vp.sizes() && w.numel() == kp.size(0) * kp.size(1), "pages and weights differ in size");
    same(budget >= 1 && budget <= INT32_MAX && recent >= 0 && recent <= budget, "budget >= 1 and 0 <= n_recent <= budget");
    same(new_len.numel() == len.numel() && kept.numel() == len.numel() * budget, "new_len is [items], kept [items][budget]");
    c.check(unlocked([&] {
      return lib.evict(c.h, kp.data_ptr(), vp.data_ptr(), kp.size(0), (float*)w.data_ptr(), (const int32_t*)table.data_ptr(), (int)table.size(1),
                       (const int32_t*)len.data_ptr(), (int)len.numel(), (int)budget, (int)recent, (const int32_t*)free_pages.data_ptr(), free_pages.numel(),
                       (int32_t*)new_table.data_ptr(), (int)new_table.size(1), (int32_t*)new_len.data_ptr(), (int32_t*)kept.data_ptr(), sz.stream());
    }), "recache_evict_rows");
    Py_RETURN_NONE;
  });
}

// the library's addresses, in the order of struct Lib
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, (Py_ssize_t)(sizeof(Lib) / sizeof(void*)), [&]() -> PyObject* {
    void** to = reinterpret_cast<void**>(&lib);
    for (Py_ssize_t i = 0; i < n; ++i) {
      to[i] = PyLong_AsVoidPtr(a[i]);
      if (PyErr_Occurred()) throw Error();
    }
    Py_RETURN_NONE;
  });
}

#define RC_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RC_METHOD(bind), RC_METHOD(encode), RC_METHOD(compact), RC_METHOD(prefill), RC_METHOD(prefill_history),
                         RC_METHOD(decode), RC_METHOD(decode_gather), RC_METHOD(compact_q8), RC_METHOD(decode_q8), RC_METHOD(decode_weighted),
                         RC_METHOD(evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  s_ws = PyUnicode_InternFromString("_ws");
  s_workspace = PyUnicode_InternFromString("workspace");
  s_check = PyUnicode_InternFromString("_check");
  s_shape = PyUnicode_InternFromString("_shape");
  return PyModule_Create(&module);
}
