// The calls of a request through the C ABI (`include/lime.h`) for torch tensors: what `binding.Lime` does per call - check the tensors,
// allocate the output, read the current stream, make the one library call - without the interpreter in between.  A request is four such
// calls with a few microseconds of GPU work each, and marshalled through ctypes they took 7 to 10 us of host time apiece, more than the
// kernels of a small batch.  Nothing is computed or kept here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <dlfcn.h>

#include "lime.h"

namespace {

decltype(&lime_lengths_to_offsets) f_offsets;
decltype(&lime_gather_history) f_gather, f_gather_ln;
decltype(&lime_encode_user) f_encode, f_encode_ln;
decltype(&lime_precompute_candidate_links) f_precompute;
decltype(&lime_score_candidates) f_score;
decltype(&lime_score_candidates_head) f_score_head;
decltype(&lime_norm_rotate) f_norm_rotate;
decltype(&lime_sequence_workspace_bytes) f_sequence_ws;
decltype(&lime_attend_history) f_attend_history;
decltype(&lime_attend_tree) f_attend_tree;
decltype(&lime_last_cuda_error) f_last_error;
PyObject* lime_error;                                            // binding.LimeError

struct Refused {};                                               // a Python error is set

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name);
    throw Refused();
  }
  return THPVariable_Unpack(o);
}
void* pointer(const at::Tensor& t) {
  if (!t.is_cuda() || !t.is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
    throw Refused();
  }
  return t.data_ptr();
}
void* pointer_or_null(PyObject* o) { return o == Py_None ? nullptr : pointer(tensor(o)); }
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int32_t integer32(int64_t v) { return static_cast<int32_t>(v); }
lime_ctx* context(PyObject* o) { return o == Py_None ? nullptr : reinterpret_cast<lime_ctx*>(integer(o)); }

// f(a..., current stream)
template <typename F, typename... A>
void call(const char* where, F f, A... a) {
  if (f == nullptr) {
    PyErr_SetString(PyExc_RuntimeError, "the library is not loaded");
    throw Refused();
  }
  lime_status s;
  void* const st = c10::cuda::getCurrentCUDAStream().stream();
  Py_BEGIN_ALLOW_THREADS
  s = f(a..., st);
  Py_END_ALLOW_THREADS
  if (s == LIME_OK) return;
  PyObject* e = PyObject_CallFunction(lime_error, "iss", static_cast<int>(s), where, s == LIME_CUDA_ERROR ? f_last_error() : "");
  if (e != nullptr) {
    PyErr_SetObject(lime_error, e);
    Py_DECREF(e);
  }
  throw Refused();
}

template <typename Body>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, Body body) {
  if (n != want) return PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, want);
  HANDLE_TH_ERRORS
  try {
    return THPVariable_Wrap(body());
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (ctx, lengths)
PyObject* lengths_to_offsets(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 2, [&] {
    const at::Tensor& len = tensor(a[1]);
    at::Tensor off = at::empty({len.numel() + 1}, len.options());
    call("lime_lengths_to_offsets", f_offsets, context(a[0]), static_cast<const int32_t*>(pointer(len)), integer32(len.numel()),
         static_cast<int32_t*>(pointer(off)));
    return off;
  });
}

// (ctx, d, table, ids, flag)
template <bool LN>
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor &table = tensor(a[2]), &ids = tensor(a[3]);
    at::Tensor out = at::empty({ids.numel(), integer(a[1])}, table.options());
    call(LN ? "lime_gather_history_normalized" : "lime_gather_history", LN ? f_gather_ln : f_gather, context(a[0]),
         static_cast<const void*>(pointer(table)), table.size(0), static_cast<const int32_t*>(pointer(ids)), ids.numel(), pointer(out),
         static_cast<int32_t*>(pointer_or_null(a[4])));
    return out;
  });
}

// (ctx, ell_c, d, hist, off, link_ctx, ws)
template <bool LN>
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const at::Tensor &hist = tensor(a[3]), &off = tensor(a[4]), &ws = tensor(a[6]);
    const int64_t B = off.numel() - 1;
    at::Tensor ls = at::empty({B, integer(a[1]), integer(a[2])}, hist.options());
    call(LN ? "lime_encode_user_normalized" : "lime_encode_user", LN ? f_encode_ln : f_encode, context(a[0]),
         static_cast<const void*>(pointer(hist)), static_cast<const int32_t*>(pointer(off)), integer32(B), hist.size(0),
         static_cast<const float*>(pointer_or_null(a[5])), pointer(ls), pointer(ws), ws.nbytes());
    return ls;
  });
}

// (ctx, ell_c, cand_emb)
PyObject* precompute(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&] {
    const at::Tensor& emb = tensor(a[2]);
    at::Tensor out = at::empty({emb.size(0), integer(a[1])}, emb.options());
    call("lime_precompute_candidate_links", f_precompute, context(a[0]), static_cast<const void*>(pointer(emb)), emb.size(0), pointer(out));
    return out;
  });
}

// (ctx, link_states, cand_w, cand_emb, C, cand_off, cand_ids, total_cands, corpus_rows, dev_flag[, ws])
template <bool HEAD>
PyObject* score(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, HEAD ? 11 : 10, [&] {
    const at::Tensor &ls = tensor(a[1]), &w = tensor(a[2]), &emb = tensor(a[3]);
    const bool by_id = a[6] != Py_None;
    const int64_t total = a[7] != Py_None ? integer(a[7]) : by_id ? tensor(a[6]).numel() : emb.size(0);
    const int64_t rows = a[8] != Py_None ? integer(a[8]) : by_id ? emb.size(0) : 0;
    at::Tensor logits = at::empty({total}, ls.options().dtype(at::kFloat));
    const void *lp = pointer(ls), *wp = pointer(w), *ep = pointer(emb);
    const int32_t *off = static_cast<const int32_t*>(pointer_or_null(a[5])), *ids = static_cast<const int32_t*>(pointer_or_null(a[6]));
    int32_t* flag = static_cast<int32_t*>(pointer_or_null(a[9]));
    float* out = static_cast<float*>(pointer(logits));
    const int32_t B = integer32(ls.size(0)), C = integer32(integer(a[4]));
    if constexpr (HEAD) {
      const at::Tensor& ws = tensor(a[10]);
      call("lime_score_candidates_head", f_score_head, context(a[0]), lp, B, wp, ep, off, C, total, ids, rows, flag, out, pointer(ws), ws.nbytes());
    } else {
      call("lime_score_candidates", f_score, context(a[0]), lp, B, wp, ep, off, C, total, ids, rows, flag, out);
    }
    return logits;
  });
}

// ---- the sequence path
[[noreturn]] void refuse(const char* name, const char* what) {
  PyErr_Format(PyExc_ValueError, "%s: expected %s", name, what);
  throw Refused();
}
// What a call of the sequence path has in common: (ctx, bf16, Hq, Hkv, d_h, q, ..); its type and device are q's.
struct Sequence {
  lime_ctx* ctx;
  int64_t Hq, Hkv, dh, n;
  const at::Tensor& q;
  c10::cuda::OptionalCUDAGuard guard;
  explicit Sequence(PyObject* const* a)
      : ctx(context(a[0])), Hq(integer(a[2])), Hkv(integer(a[3])), dh(integer(a[4])), n(0), q(tensor(a[5])) {
    if (!q.is_cuda() || q.scalar_type() != (PyObject_IsTrue(a[1]) ? at::kBFloat16 : at::kFloat) || q.dim() != 3) refuse("q", "CUDA rows of the context's type");
    n = q.size(0);
    guard.set_index(q.device().index());
  }
  struct Rows { void* p; int64_t stride; };
  Rows rows(const at::Tensor& t, int64_t heads, const char* name, int64_t want = -1) const {
    if (t.device() != q.device() || t.scalar_type() != q.scalar_type() || t.dim() != 3 || t.size(1) != heads || t.size(2) != dh)
      refuse(name, "rows [n x heads x d_h] of the type and on the device of q");
    if (want >= 0 && t.size(0) != want) refuse(name, "as many rows as the call has");
    if ((dh > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != dh)) refuse(name, "rows whose heads are contiguous");
    return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : heads * dh};
  }
  Rows rows_or_null(PyObject* o, int64_t heads, const char* name, int64_t want) const {
    return o == Py_None ? Rows{nullptr, 0} : rows(tensor(o), heads, name, want);
  }
  int32_t* ints(PyObject* o, const char* name, int64_t want = -1) const {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (t.device() != q.device() || t.scalar_type() != at::kInt || !t.is_contiguous() || (want >= 0 && t.numel() != want))
      refuse(name, "contiguous int32 on the device of q, as many as the call has");
    return static_cast<int32_t*>(t.data_ptr());
  }
  const void* vector(PyObject* o, const char* name) const {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (t.device() != q.device() || t.scalar_type() != q.scalar_type() || !t.is_contiguous() || t.numel() != dh)
      refuse(name, "d_h contiguous values of the type and on the device of q");
    return t.data_ptr();
  }
  // pages [n x rows x Hkv x d_h]; `like`: the shape they share
  const at::Tensor* pages(PyObject* o, const char* name, const at::Tensor* like = nullptr) const {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (t.device() != q.device() || t.scalar_type() != q.scalar_type() || t.dim() != 4 || t.size(2) != Hkv || t.size(3) != dh || !t.is_contiguous())
      refuse(name, "contiguous pages [n x rows x Hkv x d_h] of the type and on the device of q");
    if (like != nullptr && like->sizes() != t.sizes()) refuse(name, "the shape of cache_k");
    return &t;
  }
  int32_t users(PyObject* off) const {
    const at::Tensor& t = tensor(off);
    if (t.dim() != 1 || t.numel() < 1) refuse("off", "[users + 1]");
    return integer32(t.numel() - 1);
  }
  at::Tensor result(PyObject* o, int64_t heads) const { return o == Py_None ? at::empty({n, heads, dh}, q.options()) : tensor(o); }
  // scratch of the call's own: what it overlaps with on the GPU, or a graph that it is captured into, cannot share it
  at::Tensor scratch(int32_t B) const {
    if (f_sequence_ws == nullptr) refuse("ctx", "a loaded library");
    return at::empty({static_cast<int64_t>(f_sequence_ws(ctx, B, n))}, q.options().dtype(at::kByte));
  }
};
void* start(const at::Tensor* t) { return t == nullptr ? nullptr : t->data_ptr(); }

template <typename Body>
PyObject* guarded_object(Py_ssize_t n, Py_ssize_t want, Body body) {
  if (n != want) return PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, want);
  HANDLE_TH_ERRORS
  try {
    return body();
  } catch (const Refused&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// (ctx, bf16, Hq, Hkv, d_h, q, k, v, gamma_q, gamma_k, positions, q_out, k_out, cache_k, cache_v, slots, flag, keep_k)
PyObject* norm_rotate(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded_object(nargs, 18, [&]() -> PyObject* {
    const Sequence s(a);
    const at::Tensor *ck = s.pages(a[13], "cache_k"), *cv = s.pages(a[14], "cache_v", ck);
    const int32_t keep = PyObject_IsTrue(a[17]);
    const Sequence::Rows q = s.rows(s.q, s.Hq, "q"), k = s.rows(tensor(a[6]), s.Hkv, "k", s.n), v = s.rows_or_null(a[7], s.Hkv, "v", s.n);
    const at::Tensor q_out = s.result(a[11], s.Hq);
    at::Tensor k_out;
    if (a[12] != Py_None || ck == nullptr || keep) k_out = s.result(a[12], s.Hkv);
    const Sequence::Rows qo = s.rows(q_out, s.Hq, "q_out", s.n), ko = k_out.defined() ? s.rows(k_out, s.Hkv, "k_out", s.n) : Sequence::Rows{nullptr, 0};
    call("lime_norm_rotate", f_norm_rotate, s.ctx, static_cast<const void*>(q.p), q.stride, static_cast<const void*>(k.p), k.stride,
         static_cast<const void*>(v.p), v.stride, s.vector(a[8], "gamma_q"), s.vector(a[9], "gamma_k"),
         static_cast<const int32_t*>(s.ints(a[10], "positions", s.n)), s.n, qo.p, qo.stride, ko.p, ko.stride, start(ck), start(cv),
         ck == nullptr ? int64_t(0) : ck->size(0) * ck->size(1), static_cast<const int32_t*>(s.ints(a[15], "slots", s.n)), s.ints(a[16], "dev_flag", 1));
    PyObject *qo_obj = THPVariable_Wrap(q_out), *ko_obj = k_out.defined() ? THPVariable_Wrap(k_out) : Py_NewRef(Py_None);
    return Py_BuildValue("(NN)", qo_obj, ko_obj);
  });
}

// (ctx, bf16, Hq, Hkv, d_h, q, off, k, v, kv_off, out)
PyObject* attend_history(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 11, [&] {
    const Sequence s(a);
    const int32_t B = s.users(a[6]);
    const at::Tensor& keys = tensor(a[7]);
    const at::Tensor out = s.result(a[10], s.Hq);
    const Sequence::Rows q = s.rows(s.q, s.Hq, "q"), k = s.rows(keys, s.Hkv, "k"), v = s.rows(tensor(a[8]), s.Hkv, "v", keys.size(0)), o = s.rows(out, s.Hq, "out", s.n);
    const at::Tensor ws = s.scratch(B);
    call("lime_attend_history", f_attend_history, s.ctx, static_cast<const void*>(q.p), q.stride, static_cast<const int32_t*>(s.ints(a[6], "off")),
         static_cast<const void*>(k.p), k.stride, static_cast<const void*>(v.p), v.stride, static_cast<const int32_t*>(s.ints(a[9], "kv_off", B + 1)),
         B, s.n, keys.size(0), o.p, o.stride, ws.data_ptr(), ws.nbytes());
    return out;
  });
}

// (ctx, bf16, Hq, Hkv, d_h, q, off, parent, tree_k, tree_v, cache_k, cache_v, page_table, ctx_len, flag, out)
PyObject* attend_tree(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded(nargs, 16, [&] {
    const Sequence s(a);
    const int32_t B = s.users(a[6]);
    tensor(a[10]); tensor(a[11]);
    const at::Tensor *ck = s.pages(a[10], "cache_k"), *cv = s.pages(a[11], "cache_v", ck);
    const at::Tensor& table = tensor(a[12]);
    if (table.dim() != 2 || table.size(0) != B) refuse("page_table", "[users x pages]");
    const at::Tensor out = s.result(a[15], s.Hq);
    const Sequence::Rows q = s.rows(s.q, s.Hq, "q"), k = s.rows_or_null(a[8], s.Hkv, "tree_k", s.n), v = s.rows_or_null(a[9], s.Hkv, "tree_v", s.n), o = s.rows(out, s.Hq, "out", s.n);
    const at::Tensor ws = s.scratch(B);
    call("lime_attend_tree", f_attend_tree, s.ctx, static_cast<const void*>(q.p), q.stride, static_cast<const int32_t*>(s.ints(a[6], "off")),
         static_cast<const int32_t*>(s.ints(a[7], "parent", s.n)), static_cast<const void*>(k.p), k.stride, static_cast<const void*>(v.p), v.stride, B, s.n,
         static_cast<const void*>(start(ck)), static_cast<const void*>(start(cv)), ck->size(0), integer32(ck->size(1)),
         static_cast<const int32_t*>(s.ints(a[12], "page_table")), integer32(table.size(1)), static_cast<const int32_t*>(s.ints(a[13], "ctx_len", B)),
         s.ints(a[14], "dev_flag", 1), o.p, o.stride, ws.data_ptr(), ws.nbytes());
    return out;
  });
}

// (path of the library, LimeError)
PyObject* load(PyObject*, PyObject* args) {
  const char* path;
  PyObject* error;
  if (!PyArg_ParseTuple(args, "sO", &path, &error)) return nullptr;
  void* h = dlopen(path, RTLD_NOW);
  if (h == nullptr) return PyErr_Format(PyExc_RuntimeError, "%s", dlerror());
  bool all = true;
  auto get = [&](auto& f, const char* name) {
    f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(dlsym(h, name));
    all = all && f != nullptr;
  };
  get(f_offsets, "lime_lengths_to_offsets");
  get(f_gather, "lime_gather_history");
  get(f_gather_ln, "lime_gather_history_normalized");
  get(f_encode, "lime_encode_user");
  get(f_encode_ln, "lime_encode_user_normalized");
  get(f_precompute, "lime_precompute_candidate_links");
  get(f_score, "lime_score_candidates");
  get(f_score_head, "lime_score_candidates_head");
  get(f_norm_rotate, "lime_norm_rotate");
  get(f_sequence_ws, "lime_sequence_workspace_bytes");
  get(f_attend_history, "lime_attend_history");
  get(f_attend_tree, "lime_attend_tree");
  get(f_last_error, "lime_last_cuda_error");
  if (!all) return PyErr_Format(PyExc_RuntimeError, "%s lacks an entry point", path);
  Py_INCREF(error);
  Py_XSETREF(lime_error, error);
  Py_RETURN_NONE;
}

#define LIME_FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"load", load, METH_VARARGS, nullptr},
    LIME_FAST("lengths_to_offsets", &lengths_to_offsets),
    LIME_FAST("gather_history", &gather<false>),
    LIME_FAST("gather_history_normalized", &gather<true>),
    LIME_FAST("encode_user", &encode<false>),
    LIME_FAST("encode_user_normalized", &encode<true>),
    LIME_FAST("precompute_candidate_links", &precompute),
    LIME_FAST("score_candidates", &score<false>),
    LIME_FAST("score_candidates_head", &score<true>),
    LIME_FAST("norm_rotate", &norm_rotate),
    LIME_FAST("attend_history", &attend_history),
    LIME_FAST("attend_tree", &attend_tree),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_binding(void) {
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "made_for", LIME_MADE_FOR) < 0) Py_CLEAR(m);
  return m;
}
