// The device calls of the Python binding that a serving loop issues per layer,
// natively: the same checks as ilpc.py makes before it hands pointers over
// (tensor type, dtype, device, contiguity, shapes), then the library call.  In
// Python, the checks, the ctypes conversions and the launch took about 14 us a
// call, more than the kernels of a small batch run: an append and an attention
// call of 3 requests of 96 rows over a 64-key prefix took 30.0 us back to back,
// 8.8 with these; a host thread that stays ahead of longer kernels gains nothing.
//
// A function returns the library's code, or None with nothing called for
// whatever it does not take as it stands (another type of argument or tensor, a
// failed check; for ordinary attention a workspace still to be allocated):
// ilpc.py then takes its own path, which allocates, converts, or raises the error
// with its text.  The workspaces of differential and of tree attention, which need no
// initial contents, are allocated here on the current stream.  Nothing is kept from one call to the next but the library's entry points.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <climits>
#include <initializer_list>
#include <type_traits>

#include "../../include/ilpc.h"

namespace {

// The entry points of the library that ilpc.py has loaded (bind(), below).
decltype(&ilpc_kv_append) kv_append = nullptr;
decltype(&ilpc_rope_kv_append) rope_kv_append = nullptr;
decltype(&ilpc_attn_workspace_bytes) attn_workspace_bytes = nullptr;
decltype(&ilpc_paged_prefill_attn) prefill_attn = nullptr;
decltype(&ilpc_paged_prefill_attn_cascade) prefill_attn_cascade = nullptr;
decltype(&ilpc_extend_tables) extend_tables = nullptr;
decltype(&ilpc_release_tables) release_tables = nullptr;
decltype(&ilpc_kv_append_slots) kv_append_slots = nullptr;
decltype(&ilpc_diff_attn_workspace_bytes) diff_attn_workspace_bytes = nullptr;
decltype(&ilpc_paged_diff_attn) paged_diff_attn = nullptr;
decltype(&ilpc_tree_masks) tree_masks = nullptr;
decltype(&ilpc_tree_attn_workspace_bytes) tree_attn_workspace_bytes = nullptr;
decltype(&ilpc_paged_tree_attn) paged_tree_attn = nullptr;
decltype(&ilpc_tree_accept) tree_accept = nullptr;
decltype(&ilpc_kv_compact) kv_compact = nullptr;
decltype(&ilpc_fork_tables_drafts) fork_tables = nullptr;
decltype(&ilpc_release_shared) release_shared = nullptr;
decltype(&ilpc_copy_blocks) copy_blocks = nullptr;

constexpr int kNotHere = INT_MIN;  // what a body returns for a call it does not take

// Arguments of one call, in order; ok turns false at the first that does not fit.
struct Args {
  PyObject* const* a;
  Py_ssize_t n, i = 0;
  bool ok = true;

  PyObject* next() {
    if (i >= n) {
      ok = false;
      return Py_None;
    }
    return a[i++];
  }
  // A plain contiguous GPU tensor of this type and rank (nullptr otherwise).
  const at::Tensor* tensor(at::ScalarType type, int64_t dim) {
    PyObject* o = next();
    if (!ok || !THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || t.dim() != dim || !t.is_contiguous()) {
      ok = false;
      return nullptr;
    }
    return &t;
  }
  const at::Tensor* tensor_or_none(at::ScalarType type, int64_t dim) {
    if (i < n && a[i] == Py_None) {
      ++i;
      return nullptr;
    }
    return tensor(type, dim);
  }
  int32_t integer() {
    PyObject* o = next();
    if (!ok || !PyLong_CheckExact(o)) {
      ok = false;
      return 0;
    }
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v != int32_t(v)) ok = false;
    return int32_t(v);
  }
  float real() {
    PyObject* o = next();
    if (!ok || !PyFloat_Check(o)) {
      ok = false;
      return 0.f;
    }
    return float(PyFloat_AS_DOUBLE(o));
  }
};

// The stream of a call: a torch stream object, or None for the current
// device's current stream; and its device's index.
bool stream_of(PyObject* o, void** stream, int* device) {
  if (o == Py_None) {
    const auto s = c10::hip::getCurrentHIPStream();
    *stream = s.stream();
    *device = s.device_index();
    return true;
  }
  PyObject* p = PyObject_GetAttrString(o, "cuda_stream");
  PyObject* d = p ? PyObject_GetAttrString(o, "device_index") : nullptr;
  bool ok = p && d && PyLong_Check(p) && PyLong_Check(d);
  if (ok) {
    *stream = PyLong_AsVoidPtr(p);
    *device = int(PyLong_AsLong(d));
    ok = !PyErr_Occurred();
  }
  Py_XDECREF(p);
  Py_XDECREF(d);
  return ok;
}

uint16_t* bf16(const at::Tensor* t) { return static_cast<uint16_t*>(t->data_ptr()); }
int32_t* i32(const at::Tensor* t) { return static_cast<int32_t*>(t->data_ptr()); }

// Pools [NB, Hkv, 16, D] and [NB, Hkv, D, 16] that fit each other.
bool pools_fit(const at::Tensor& k, const at::Tensor& v) {
  return v.size(0) == k.size(0) && v.size(1) == k.size(1) && v.size(2) == k.size(3) && v.size(3) == k.size(2);
}

// Runs a call body: its code, or None.  What it throws (torch's checks do) or
// leaves as a Python error comes before the library call and means None.
template <class F>
PyObject* guarded(F&& body) {
  int rc = kNotHere;
  try {
    rc = body();
  } catch (const std::exception&) {
  }
  PyErr_Clear();
  if (rc == kNotHere) Py_RETURN_NONE;
  return PyLong_FromLong(rc);
}

// The library call, without the interpreter's lock (the arguments are evaluated with it: data_ptr() may throw).
template <class... P, class... A>
int call(int (*fn)(P...), A... args) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = fn(args...);
  Py_END_ALLOW_THREADS;
  return rc;
}

// bind(addresses of the entry points above, in their order)
PyObject* py_bind(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  constexpr int kEntries = 18;
  void* p[kEntries];
  if (n != kEntries) {
    PyErr_Format(PyExc_TypeError, "bind() takes %d addresses", kEntries);
    return nullptr;
  }
  for (int i = 0; i < kEntries; ++i) p[i] = PyLong_AsVoidPtr(argv[i]);
  if (PyErr_Occurred()) return nullptr;
  int i = 0;
  auto set = [&](auto& fn) { fn = reinterpret_cast<std::decay_t<decltype(fn)>>(p[i++]); };
  set(kv_append), set(rope_kv_append), set(attn_workspace_bytes), set(prefill_attn), set(prefill_attn_cascade);
  set(extend_tables), set(release_tables), set(kv_append_slots), set(diff_attn_workspace_bytes), set(paged_diff_attn);
  set(tree_masks), set(tree_attn_workspace_bytes), set(paged_tree_attn), set(tree_accept), set(kv_compact);
  set(fork_tables), set(release_shared), set(copy_blocks);
  Py_RETURN_NONE;
}

// kv_append(k_new, v_new, k_pool, v_pool, block_tables, cu_new, start_pos, max_new, stream)
PyObject* py_kv_append(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    const at::Tensor *k = a.tensor(at::kBFloat16, 3), *v = a.tensor(at::kBFloat16, 3),
                     *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4), *bt = a.tensor(at::kInt, 2),
                     *cu = a.tensor(at::kInt, 1), *sp = a.tensor(at::kInt, 1);
    const int32_t max_new = a.integer();
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t NB = kp->size(0), Hkv = kp->size(1), bs = kp->size(2), D = kp->size(3), B = cu->size(0) - 1;
    if (!pools_fit(*kp, *vp) || k->size(1) != Hkv || k->size(2) != D || v->sizes() != k->sizes() ||
        bt->size(0) != B || sp->size(0) != B)
      return kNotHere;
    void* s;
    int dev;
    if (!stream_of(so, &s, &dev)) return kNotHere;
    return call(kv_append, bf16(k), bf16(v), bf16(kp), bf16(vp), int32_t(NB), i32(bt), int32_t(bt->size(1)), i32(cu),
                i32(sp), int32_t(B), max_new, int32_t(Hkv), int32_t(D), int32_t(bs), s);
  });
}

// rope_kv_append(q, q_out, k_new, v_new, k_pool, v_pool, block_tables, cu_new, start_pos, max_new, inv_freq, stream)
PyObject* py_rope_kv_append(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    const at::Tensor *q = a.tensor_or_none(at::kBFloat16, 3), *qo = a.tensor_or_none(at::kBFloat16, 3),
                     *k = a.tensor(at::kBFloat16, 3), *v = a.tensor(at::kBFloat16, 3),
                     *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4), *bt = a.tensor(at::kInt, 2),
                     *cu = a.tensor(at::kInt, 1), *sp = a.tensor(at::kInt, 1);
    const int32_t max_new = a.integer();
    const at::Tensor* fr = a.tensor(at::kFloat, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t NB = kp->size(0), Hkv = kp->size(1), bs = kp->size(2), D = kp->size(3), B = cu->size(0) - 1;
    if (!pools_fit(*kp, *vp) || k->size(1) != Hkv || k->size(2) != D || v->sizes() != k->sizes() ||
        !q != !qo || (q && (q->size(0) != k->size(0) || q->size(2) != D || qo->sizes() != q->sizes())) ||
        fr->size(0) != D / 2 || bt->size(0) != B || sp->size(0) != B)
      return kNotHere;
    void* s;
    int dev;
    if (!stream_of(so, &s, &dev)) return kNotHere;
    return call(rope_kv_append, q ? bf16(q) : nullptr, q ? bf16(qo) : nullptr, int32_t(q ? q->size(1) : Hkv),
                bf16(k), bf16(v), bf16(kp), bf16(vp), int32_t(NB), i32(bt), int32_t(bt->size(1)), i32(cu), i32(sp),
                int32_t(B), max_new, int32_t(Hkv), int32_t(D), int32_t(bs), static_cast<float*>(fr->data_ptr()), s);
  });
}

struct Attn {
  const at::Tensor *q, *kp, *vp, *bt, *cu, *L;
  int32_t max_q;
  int64_t B;

  bool read(Args& a) {
    q = a.tensor(at::kBFloat16, 3), kp = a.tensor(at::kBFloat16, 4), vp = a.tensor(at::kBFloat16, 4);
    bt = a.tensor(at::kInt, 2), cu = a.tensor(at::kInt, 1), L = a.tensor(at::kInt, 1);
    max_q = a.integer();
    if (!a.ok) return false;
    B = cu->size(0) - 1;
    return q->size(2) == kp->size(3) && pools_fit(*kp, *vp) && bt->size(0) == B && L->size(0) == B;
  }
};

// paged_prefill_attn(q, k_pool, v_pool, block_tables, cu_q, seq_lens, max_q_len, scale, out, workspace, stream,
//                    workspaces kept by (device index, stream))
PyObject* py_prefill_attn(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    Attn t;
    if (!t.read(a)) return kNotHere;
    const float scale = a.real();
    const at::Tensor* out = a.tensor(at::kBFloat16, 3);
    PyObject *wo = a.next(), *so = a.next(), *kept = a.next();
    if (!a.ok || out->sizes() != t.q->sizes() || !PyDict_CheckExact(kept)) return kNotHere;
    void* s;
    int dev;
    if (!stream_of(so, &s, &dev)) return kNotHere;
    const int32_t Hq = int32_t(t.q->size(1)), Hkv = int32_t(t.kp->size(1)), D = int32_t(t.kp->size(3));
    if (wo == Py_None) {
      // the kept buffer of this stream, where it is there and large enough
      size_t need = 0;
      if (t.q->device().index() != dev || attn_workspace_bytes(int32_t(t.B), t.max_q, Hq, Hkv, D, &need) != ILPC_OK)
        return kNotHere;
      PyObject* key = Py_BuildValue("(iN)", dev, PyLong_FromVoidPtr(s));
      wo = key ? PyDict_GetItemWithError(kept, key) : nullptr;  // (borrowed: the dictionary holds it)
      Py_XDECREF(key);
      if (!wo || !THPVariable_CheckExact(wo) || size_t(THPVariable_Unpack(wo).numel()) < need) return kNotHere;
    }
    PyObject* one[1] = {wo};
    Args w{one, 1};
    const at::Tensor* ws = w.tensor(at::kByte, 1);
    if (!w.ok) return kNotHere;
    const at::Tensor hold = *ws;  // (another thread may replace the kept buffer once the lock is let go)
    return call(prefill_attn, bf16(t.q), bf16(t.kp), bf16(t.vp), int32_t(t.kp->size(0)), i32(t.bt),
                int32_t(t.bt->size(1)), i32(t.cu), i32(t.L), int32_t(t.B), t.max_q, Hq, Hkv, D,
                int32_t(t.kp->size(2)), scale, bf16(out), hold.data_ptr(), size_t(hold.numel()), s);
  });
}

// paged_prefill_attn_cascade(q, k_pool, v_pool, block_tables, cu_q, seq_lens, max_q_len, shared_len, scale, out,
//                            workspace, stream)
PyObject* py_prefill_attn_cascade(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    Attn t;
    if (!t.read(a)) return kNotHere;
    const int32_t shared = a.integer();
    const float scale = a.real();
    const at::Tensor *out = a.tensor(at::kBFloat16, 3), *ws = a.tensor(at::kByte, 1);
    PyObject* so = a.next();
    if (!a.ok || out->sizes() != t.q->sizes()) return kNotHere;
    void* s;
    int dev;
    if (!stream_of(so, &s, &dev)) return kNotHere;
    return call(prefill_attn_cascade, bf16(t.q), bf16(t.kp), bf16(t.vp), int32_t(t.kp->size(0)), i32(t.bt),
                int32_t(t.bt->size(1)), i32(t.cu), i32(t.L), int32_t(t.B), t.max_q, int32_t(t.q->size(1)),
                int32_t(t.kp->size(1)), int32_t(t.kp->size(3)), int32_t(t.kp->size(2)), shared, scale, bf16(out),
                ws->data_ptr(), size_t(ws->numel()), s);
  });
}

// Tensors of one call: all on the stream's device, which is the current one (the
// general path makes another one current), the stream's pointer in *s.
bool placed(std::initializer_list<const at::Tensor*> tensors, PyObject* so, void** s) {
  int dev;
  if (!stream_of(so, s, &dev) || dev != c10::hip::current_device()) return false;
  for (const at::Tensor* t : tensors)
    if (t && t->device().index() != dev) return false;
  return true;
}

struct Span {
  const char *from, *to;
  explicit Span(const at::Tensor* t)
      : from(static_cast<const char*>(t->data_ptr())), to(from + t->numel() * t->element_size()) {}
  bool meets(const Span& o) const { return from < o.to && o.from < to && from < to && o.from < o.to; }
};

// Whether outputs share memory with an input or with each other.
bool apart(std::initializer_list<const at::Tensor*> outputs, std::initializer_list<const at::Tensor*> inputs) {
  for (auto a = outputs.begin(); a != outputs.end(); ++a) {
    const Span s(*a);
    for (auto b = a + 1; b != outputs.end(); ++b)
      if (s.meets(Span(*b))) return false;
    for (const at::Tensor* b : inputs)
      if (b && s.meets(Span(b))) return false;
  }
  return true;
}

// extend_tables(block_tables, start_pos, new_lens, free_ids, taken, seq_lens, cu_q, cu_blocks, slot_map, taken_out,
//               status, num_blocks, stream)
PyObject* py_extend_tables(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    auto ints = [&](int64_t dim) { return a.tensor(at::kInt, dim); };
    const at::Tensor *bt = ints(2), *start = ints(1), *add = ints(1), *free = ints(1), *taken = ints(1), *seq = ints(1),
                     *cu = ints(1), *cb = ints(1), *slots = ints(1), *out = ints(1), *status = ints(1);
    const int32_t nb = a.integer();
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = start->size(0);
    if (bt->size(0) != B || add->size(0) != B || seq->size(0) != B || cu->size(0) != B + 1 || cb->size(0) != B + 1 ||
        taken->size(0) != 1 || out->size(0) != 1 || status->size(0) != 1)
      return kNotHere;
    if (!apart({bt, cu, cb, slots, status, seq, out},
               {add, free, seq->data_ptr() == start->data_ptr() ? nullptr : start,
                out->data_ptr() == taken->data_ptr() ? nullptr : taken}))
      return kNotHere;
    void* s;
    if (!placed({bt, start, add, free, taken, seq, cu, cb, slots, out, status}, so, &s)) return kNotHere;
    return call(extend_tables, i32(bt), int32_t(bt->size(1)), int32_t(B), i32(start), i32(add), i32(free),
                int32_t(free->size(0)), i32(taken), nb, i32(seq), i32(cu), i32(cb), i32(slots),
                int32_t(slots->size(0)), i32(out), i32(status), s);
  });
}

// release_tables(block_tables, first_block, seq_lens, free_ids, taken, cu_blocks, taken_out, status, stream)
PyObject* py_release_tables(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    auto ints = [&](int64_t dim) { return a.tensor(at::kInt, dim); };
    const at::Tensor *bt = ints(2), *first = ints(1), *seq = ints(1), *free = ints(1), *taken = ints(1), *cb = ints(1),
                     *out = ints(1), *status = ints(1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = first->size(0);
    if (bt->size(0) != B || seq->size(0) != B || cb->size(0) != B + 1 || taken->size(0) != 1 || out->size(0) != 1 ||
        status->size(0) != 1)
      return kNotHere;
    if (!apart({free, cb, status, out},
               {bt, first, seq, out->data_ptr() == taken->data_ptr() ? nullptr : taken}))
      return kNotHere;
    void* s;
    if (!placed({bt, first, seq, free, taken, cb, out, status}, so, &s)) return kNotHere;
    return call(release_tables, i32(bt), int32_t(bt->size(1)), int32_t(B), i32(first), i32(seq), i32(free),
                int32_t(free->size(0)), i32(taken), i32(cb), i32(out), i32(status), s);
  });
}

// bf16 rows [n, H, D], each contiguous, *stride elements apart (nullptr: others).
const at::Tensor* rows(Args& a, int64_t* stride) {
  PyObject* o = a.next();
  a.ok = a.ok && THPVariable_CheckExact(o);
  if (!a.ok) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  a.ok = t.is_cuda() && t.scalar_type() == at::kBFloat16 && t.layout() == at::kStrided && t.dim() == 3 &&
         (t.numel() == 0 || (t.stride(2) == 1 && (t.size(1) <= 1 || t.stride(1) == t.size(2))));
  if (!a.ok) return nullptr;
  *stride = t.size(0) > 1 ? t.stride(0) : t.size(1) * t.size(2);
  return &t;
}

// kv_append_slots(k_new, v_new, k_pool, v_pool, slot_map, stream)
PyObject* py_kv_append_slots(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    int64_t ks = 0, vs = 0;
    const at::Tensor *k = rows(a, &ks), *v = rows(a, &vs), *kp = a.tensor(at::kBFloat16, 4),
                     *vp = a.tensor(at::kBFloat16, 4), *slots = a.tensor(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t Hkv = kp->size(1), D = kp->size(3);
    if (!pools_fit(*kp, *vp) || k->size(1) != Hkv || k->size(2) != D || v->sizes() != k->sizes() ||
        slots->size(0) != k->size(0))
      return kNotHere;
    void* s;
    if (!placed({k, v, kp, vp, slots}, so, &s)) return kNotHere;
    return call(kv_append_slots, bf16(k), ks, bf16(v), vs, bf16(kp), bf16(vp), int32_t(kp->size(0)), i32(slots),
                int32_t(slots->size(0)), int32_t(Hkv), int32_t(D), int32_t(kp->size(2)), s);
  });
}

// paged_diff_attn(q, k_pool, v_pool, block_tables, cu_q, seq_lens, max_q_len, scale, lam, out, norm_weight, norm_eps,
//                 out_scale, layout, workspace, stream)
PyObject* py_paged_diff_attn(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    int64_t qs = 0;
    const at::Tensor *q = rows(a, &qs), *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4),
                     *bt = a.tensor(at::kInt, 2), *cu = a.tensor(at::kInt, 1), *L = a.tensor(at::kInt, 1);
    const int32_t max_q = a.integer();
    const float scale = a.real();
    const at::Tensor *lam = a.tensor(at::kFloat, 1), *out = a.tensor(at::kBFloat16, 3),
                     *w = a.tensor_or_none(at::kFloat, 1);
    const float eps = a.real(), out_scale = a.real();
    const int32_t layout = a.integer();
    const at::Tensor* ws = a.tensor_or_none(at::kByte, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = cu->size(0) - 1, Hq = q->size(1), Hkv = kp->size(1), D = kp->size(3);
    if (!pools_fit(*kp, *vp) || q->size(2) != D || out->sizes() != q->sizes() || bt->size(0) != B ||
        L->size(0) != B || lam->size(0) != Hq || (w && w->size(0) != D))
      return kNotHere;
    void* s;
    if (!placed({q, kp, vp, bt, cu, L, lam, out, w, ws}, so, &s)) return kNotHere;
    at::Tensor own;  // the call's scratch, from the current stream's memory
    if (!ws) {
      size_t need = 0;
      if (diff_attn_workspace_bytes(int32_t(B), max_q, int32_t(Hq), int32_t(Hkv), int32_t(D), int32_t(bt->size(1)),
                                    &need) != ILPC_OK ||
          (need && so != Py_None))
        return kNotHere;
      if (need) own = at::empty({int64_t(need)}, q->options().dtype(at::kByte));
    }
    const at::Tensor* scratch = ws ? ws : own.defined() ? &own : nullptr;
    return call(paged_diff_attn, bf16(q), qs, int32_t(q->size(0)), bf16(kp), bf16(vp), int32_t(kp->size(0)), i32(bt),
                int32_t(bt->size(1)), i32(cu), i32(L), int32_t(B), max_q, int32_t(Hq), int32_t(Hkv), int32_t(D),
                int32_t(kp->size(2)), scale, layout, static_cast<float*>(lam->data_ptr()),
                w ? static_cast<float*>(w->data_ptr()) : nullptr, eps, out_scale, bf16(out),
                scratch ? scratch->data_ptr() : nullptr, scratch ? size_t(scratch->numel()) : size_t(0), s);
  });
}

uint64_t* u64(const at::Tensor* t) { return static_cast<uint64_t*>(t->data_ptr()); }

// tree_masks(parents, cu_q, masks, positions, start_pos, stream)
PyObject* py_tree_masks(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    const at::Tensor *par = a.tensor(at::kInt, 1), *cu = a.tensor(at::kInt, 1), *m = a.tensor(at::kLong, 2),
                     *pos = a.tensor_or_none(at::kInt, 1), *start = a.tensor_or_none(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t rows = par->size(0), B = cu->size(0) - 1;
    if (m->size(0) != rows || (pos && pos->size(0) != rows) || (start && start->size(0) != B)) return kNotHere;
    if (pos ? !apart({m, pos}, {par, cu, start}) : !apart({m}, {par, cu, start})) return kNotHere;
    void* s;
    if (!placed({par, cu, m, pos, start}, so, &s)) return kNotHere;
    return call(tree_masks, i32(par), i32(cu), start ? i32(start) : nullptr, int32_t(B), int32_t(rows),
                int32_t(m->size(1)), u64(m), pos ? i32(pos) : nullptr, s);
  });
}

// paged_tree_attn(q, k_pool, v_pool, block_tables, cu_q, seq_lens, max_q_len, scale, masks, out, workspace, stream)
PyObject* py_paged_tree_attn(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    int64_t qs = 0;
    const at::Tensor *q = rows(a, &qs), *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4),
                     *bt = a.tensor(at::kInt, 2), *cu = a.tensor(at::kInt, 1), *L = a.tensor(at::kInt, 1);
    const int32_t max_q = a.integer();
    const float scale = a.real();
    const at::Tensor *m = a.tensor(at::kLong, 2), *out = a.tensor(at::kBFloat16, 3),
                     *ws = a.tensor_or_none(at::kByte, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = cu->size(0) - 1, Hq = q->size(1), Hkv = kp->size(1), D = kp->size(3);
    if (!pools_fit(*kp, *vp) || q->size(2) != D || out->sizes() != q->sizes() || bt->size(0) != B ||
        L->size(0) != B || m->size(0) != q->size(0))
      return kNotHere;
    void* s;
    if (!placed({q, kp, vp, bt, cu, L, m, out, ws}, so, &s)) return kNotHere;
    at::Tensor own;  // the call's scratch, from the current stream's memory
    if (!ws) {
      size_t need = 0;
      if (tree_attn_workspace_bytes(int32_t(B), max_q, int32_t(Hq), int32_t(Hkv), int32_t(D), int32_t(bt->size(1)),
                                    &need) != ILPC_OK ||
          (need && so != Py_None))
        return kNotHere;
      if (need) own = at::empty({int64_t(need)}, q->options().dtype(at::kByte));
    }
    const at::Tensor* scratch = ws ? ws : own.defined() ? &own : nullptr;
    return call(paged_tree_attn, bf16(q), qs, int32_t(q->size(0)), bf16(kp), bf16(vp), int32_t(kp->size(0)), i32(bt),
                int32_t(bt->size(1)), i32(cu), i32(L), int32_t(B), max_q, int32_t(Hq), int32_t(Hkv), int32_t(D),
                int32_t(kp->size(2)), scale, u64(m), int32_t(m->size(1)), bf16(out),
                scratch ? scratch->data_ptr() : nullptr, scratch ? size_t(scratch->numel()) : size_t(0), s);
  });
}

// tree_accept(parents, tokens, targets, cu_q, start_pos, path, n_accepted, next_tokens, kept_lens, kept_blocks,
//             root_targets, stream)
PyObject* py_tree_accept(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    auto ints = [&]() { return a.tensor(at::kInt, 1); };
    const at::Tensor *par = ints(), *tok = ints(), *pick = ints(), *cu = ints(), *start = ints(), *path = ints(),
                     *count = ints(), *next = ints(), *lens = ints(), *blocks = ints(),
                     *root = a.tensor_or_none(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t N = par->size(0), B = start->size(0);
    if (tok->size(0) != N || pick->size(0) != N || path->size(0) != N || cu->size(0) != B + 1 || count->size(0) != B ||
        next->size(0) != B || lens->size(0) != B || blocks->size(0) != B || (root && root->size(0) != B))
      return kNotHere;
    if (!apart({path, count, next, lens, blocks}, {par, tok, pick, cu, start, root})) return kNotHere;
    void* s;
    if (!placed({par, tok, pick, cu, start, path, count, next, lens, blocks, root}, so, &s)) return kNotHere;
    return call(tree_accept, i32(par), i32(tok), i32(pick), root ? i32(root) : nullptr, i32(cu), i32(start),
                int32_t(B), int32_t(N), i32(path), i32(count), i32(next), i32(lens), i32(blocks), s);
  });
}

// kv_compact(k_pool, v_pool, block_tables, cu_q, start_pos, path, n_accepted, stream)
PyObject* py_kv_compact(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    const at::Tensor *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4), *bt = a.tensor(at::kInt, 2),
                     *cu = a.tensor(at::kInt, 1), *start = a.tensor(at::kInt, 1), *path = a.tensor(at::kInt, 1),
                     *count = a.tensor(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = start->size(0);
    if (!pools_fit(*kp, *vp) || bt->size(0) != B || cu->size(0) != B + 1 || count->size(0) != B) return kNotHere;
    void* s;
    if (!placed({kp, vp, bt, cu, start, path, count}, so, &s)) return kNotHere;
    return call(kv_compact, bf16(kp), bf16(vp), int32_t(kp->size(0)), i32(bt), int32_t(bt->size(1)), i32(cu),
                i32(start), int32_t(B), int32_t(path->size(0)), i32(path), i32(count), int32_t(kp->size(1)),
                int32_t(kp->size(3)), int32_t(kp->size(2)), s);
  });
}

// Whether these are the hold counts of blocks first .. num_blocks - 1.
bool holds_fit(const at::Tensor& holds, int64_t num_blocks, int64_t first) {
  const int64_t held = num_blocks - first;
  return first >= 0 && held >= 0 && holds.size(0) == held + (held + 31) / 32;
}

// fork_tables(block_tables, seq_lens, sources, holds, first_id, free_ids, taken, copy_src, copy_dst, taken_out, status,
//             num_blocks, start_pos, stream)
PyObject* py_fork_tables(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    auto ints = [&](int64_t dim) { return a.tensor(at::kInt, dim); };
    const at::Tensor *bt = ints(2), *seq = ints(1), *src = ints(1), *holds = ints(1);
    const int32_t first = a.integer();
    const at::Tensor *free = ints(1), *taken = ints(1), *from = ints(1), *to = ints(1), *out = ints(1),
                     *status = ints(1);
    const int32_t nb = a.integer();
    const at::Tensor* start = a.tensor_or_none(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = src->size(0);
    if (bt->size(0) != B || seq->size(0) != B || from->size(0) != B || to->size(0) != B || taken->size(0) != 1 ||
        out->size(0) != 1 || status->size(0) != 1 || (start && start->size(0) != B) ||
        !holds_fit(*holds, nb, first))
      return kNotHere;
    const at::Tensor* had = out->data_ptr() == taken->data_ptr() ? nullptr : taken;
    if (start ? !apart({bt, seq, holds, from, to, status, out, start}, {src, free, had})
              : !apart({bt, seq, holds, from, to, status, out}, {src, free, had}))
      return kNotHere;
    void* s;
    if (!placed({bt, seq, src, holds, free, taken, from, to, out, status, start}, so, &s)) return kNotHere;
    return call(fork_tables, i32(bt), int32_t(bt->size(1)), int32_t(B), i32(seq), i32(src), i32(holds), first,
                i32(free), int32_t(free->size(0)), i32(taken), nb, i32(from), i32(to), start ? i32(start) : nullptr,
                i32(out), i32(status), s);
  });
}

// release_shared(block_tables, seq_lens, holds, first_id, free_ids, taken, taken_out, status, num_blocks, stream)
PyObject* py_release_shared(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    auto ints = [&](int64_t dim) { return a.tensor(at::kInt, dim); };
    const at::Tensor *bt = ints(2), *seq = ints(1), *holds = ints(1);
    const int32_t first = a.integer();
    const at::Tensor *free = ints(1), *taken = ints(1), *out = ints(1), *status = ints(1);
    const int32_t nb = a.integer();
    PyObject* so = a.next();
    if (!a.ok) return kNotHere;
    const int64_t B = seq->size(0);
    if (bt->size(0) != B || taken->size(0) != 1 || out->size(0) != 1 || status->size(0) != 1 ||
        !holds_fit(*holds, nb, first))
      return kNotHere;
    if (!apart({holds, free, status, out}, {bt, seq, out->data_ptr() == taken->data_ptr() ? nullptr : taken}))
      return kNotHere;
    void* s;
    if (!placed({bt, seq, holds, free, taken, out, status}, so, &s)) return kNotHere;
    return call(release_shared, i32(bt), int32_t(bt->size(1)), int32_t(B), i32(seq), i32(holds), first, i32(free),
                int32_t(free->size(0)), i32(taken), nb, i32(out), i32(status), s);
  });
}

// copy_blocks(k_pool, v_pool, src, dst, stream)
PyObject* py_copy_blocks(PyObject*, PyObject* const* argv, Py_ssize_t n) {
  return guarded([&]() -> int {
    Args a{argv, n};
    const at::Tensor *kp = a.tensor(at::kBFloat16, 4), *vp = a.tensor(at::kBFloat16, 4), *src = a.tensor(at::kInt, 1),
                     *dst = a.tensor(at::kInt, 1);
    PyObject* so = a.next();
    if (!a.ok || !pools_fit(*kp, *vp) || dst->size(0) != src->size(0)) return kNotHere;
    void* s;
    if (!placed({kp, vp, src, dst}, so, &s)) return kNotHere;
    return call(copy_blocks, bf16(kp), bf16(vp), int32_t(kp->size(0)), i32(src), i32(dst), int32_t(src->size(0)),
                int32_t(kp->size(1)), int32_t(kp->size(3)), int32_t(kp->size(2)), s);
  });
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST("bind", py_bind),
                         FAST("kv_append", py_kv_append), FAST("rope_kv_append", py_rope_kv_append),
                         FAST("paged_prefill_attn", py_prefill_attn),
                         FAST("paged_prefill_attn_cascade", py_prefill_attn_cascade),
                         FAST("extend_tables", py_extend_tables), FAST("release_tables", py_release_tables),
                         FAST("kv_append_slots", py_kv_append_slots), FAST("paged_diff_attn", py_paged_diff_attn),
                         FAST("tree_masks", py_tree_masks), FAST("paged_tree_attn", py_paged_tree_attn),
                         FAST("tree_accept", py_tree_accept), FAST("kv_compact", py_kv_compact),
                         FAST("fork_tables", py_fork_tables), FAST("release_shared", py_release_shared),
                         FAST("copy_blocks", py_copy_blocks),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
