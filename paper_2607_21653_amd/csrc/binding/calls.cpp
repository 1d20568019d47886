// The Python calls of sparse attention and its cache's upkeep, from tensors to the C entries. These take 3 to 8 us on the
// GPU where they are small, and asking 6 tensors for what a call needs took as long in Python; here it is done in one.
//
// Every call returns None where it does not take the arguments (a wrong type, shape, device or stride), having enqueued
// nothing: the Python function then finds the words for it. What a C entry refuses is raised as a MoltError. A workspace
// that the caller did not give, or a smaller one, is made here, and the outputs are, once the entry's checks of the sizes
// let them pass. The entries come from the loaded library (set_entries).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../../include/molt.h"
#include "sizes.h"

namespace {

PyObject* error_class;
decltype(&molt_last_error) last_error;
decltype(&molt_plan_blocks) plan_entry;
decltype(&molt_plan_blocks_workspace_size) plan_size;
decltype(&molt_kv_write) write_entry;
decltype(&molt_key_bounds_update) update_entry;
decltype(&molt_key_bounds_read) read_entry;
decltype(&molt_select_blocks) select_entry;
decltype(&molt_select_blocks_workspace_size) select_size;
decltype(&molt_paged_attention_blocks) attend_entry;
decltype(&molt_paged_attention_blocks_workspace_size) attend_size;
decltype(&molt_plan_blocks_takes) plan_takes;
decltype(&molt_key_bounds_read_takes) read_takes;
decltype(&molt_select_blocks_takes) select_takes;
decltype(&molt_paged_attention_blocks_takes) attend_takes;

// Arguments in turn; `fine` ends false where one is not what a call takes
struct Args {
  PyObject* const* at;
  bool fine = true;
  const at::Tensor* tensor() {
    PyObject* o = *at++;
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    fine = false;
    return nullptr;
  }
  const at::Tensor* tensor_or_none() {
    if (*at != Py_None) return tensor();
    ++at;
    return nullptr;
  }
  // of any type of whole numbers; a tensor is none, which would have to be waited for
  int number() {
    PyObject* o = *at++;
    long v = -1;
    if (PyLong_Check(o)) {
      v = PyLong_AsLong(o);
    } else if (PyIndex_Check(o) && !THPVariable_Check(o)) {
      if (PyObject* whole = PyNumber_Index(o)) {
        v = PyLong_AsLong(whole);
        Py_DECREF(whole);
      }
    }
    if (v < 0 || v > 0x7fffffff) {
      PyErr_Clear();
      fine = false;
    }
    return int(v);
  }
  molt_stream_t stream() {
    void* v = PyLong_Check(*at) ? PyLong_AsVoidPtr(*at) : nullptr;
    fine = fine && PyLong_Check(*at);
    ++at;
    return static_cast<molt_stream_t>(v);
  }
};

bool on(const at::Tensor& t, int dev) { return t.is_cuda() && t.get_device() == dev; }
bool whole(const at::Tensor& t, at::ScalarType type, int dev) {
  return t.scalar_type() == type && on(t, dev) && t.is_contiguous();
}
bool ints(const at::Tensor& t, int64_t n, int dev) { return whole(t, at::kInt, dev) && t.dim() == 1 && t.size(0) == n; }
bool table(const at::Tensor& t, int dev) {
  return whole(t, at::kInt, dev) && t.dim() == 2 && t.size(0) < (1l << 31) && t.size(1) < (1l << 31);
}
bool floats(at::ScalarType t) { return t == at::kBFloat16 || t == at::kFloat; }
molt_dtype code(at::ScalarType t) { return t == at::kFloat ? MOLT_F32 : MOLT_BF16; }
const int32_t* i32(const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->const_data_ptr()) : nullptr; }
int32_t* i32_out(const at::Tensor& t) { return static_cast<int32_t*>(t.data_ptr()); }
bool keys(const at::Tensor& k, int dev) {
  return floats(k.scalar_type()) && whole(k, k.scalar_type(), dev) && k.dim() == 4 && k.size(2) == 16;
}
bool values_of(const at::Tensor& k, const at::Tensor& v, int dev) {
  return whole(v, k.scalar_type(), dev) && v.dim() == 4 && v.size(0) == k.size(0) && v.size(1) == k.size(1) &&
         v.size(2) == k.size(3) && v.size(3) == 16;
}
bool bounds_of(const at::Tensor& b, int dev) {
  return whole(b, at::kByte, dev) && b.dim() == 3 && b.size(2) > 16 && b.size(2) % 2 == 0;
}
// rows [T, H, D] whose heads are contiguous; their stride
bool rows(const at::Tensor& t, at::ScalarType type, int64_t T, int64_t H, int64_t D, int dev, int64_t& stride) {
  if (t.scalar_type() != type || !on(t, dev) || t.dim() != 3 || t.size(0) != T || t.size(1) != H || t.size(2) != D ||
      t.stride(2) != 1 || (H > 1 && t.stride(1) != D) || (T > 1 && t.stride(0) < H * D))
    return false;
  stride = T > 1 ? t.stride(0) : H * D;
  return true;
}
bool room(const at::Tensor* ws, int dev, void*& at, size_t& bytes) {
  at = nullptr;
  bytes = 0;
  if (!ws) return true;
  if (!on(*ws, dev) || !ws->is_contiguous()) return false;
  at = ws->data_ptr();
  bytes = ws->nbytes();
  return true;
}

at::Tensor bytes_like(const at::Tensor& t, size_t n) { return at::empty({int64_t(n)}, t.options().dtype(at::kByte)); }

#define TAKE(cond) do { if (!(cond)) Py_RETURN_NONE; } while (0)
#define RUN(name, expr) \
  do { \
    if (const int st = (expr)) { \
      PyErr_Format(error_class, name " returned %d: %s", st, last_error()); \
      return nullptr; \
    } \
  } while (0)
#define CALL(name, count) \
  PyObject* name(PyObject*, PyObject* const* argv, Py_ssize_t argc) { \
    HANDLE_TH_ERRORS \
    if (argc != count) { PyErr_SetString(PyExc_TypeError, #name " takes " #count " arguments"); return nullptr; } \
    Args in{argv};
#define END_CALL END_HANDLE_TH_ERRORS }

CALL(plan, 9)  // block_tables, n_blocks, context_lens, n_new, pool, n, n_shared, device, stream
  const at::Tensor *bt = in.tensor(), *have = in.tensor(), *ctx = in.tensor(), *fresh = in.tensor(), *pool = in.tensor();
  const int n = in.number();
  const at::Tensor* shared = in.tensor_or_none();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  TAKE(in.fine && n > 0 && table(*bt, dev));
  const int64_t B = bt->size(0), cap = pool->numel() - 2;
  TAKE(ints(*have, B, dev) && ints(*ctx, B, dev) && ints(*fresh, B, dev) && cap > 0 && cap < (1l << 31) &&
       ints(*pool, cap + 2, dev) && (!shared || ints(*shared, B, dev)));
  RUN("molt_plan_blocks", plan_takes(int(B), n, int(bt->size(1)), int(cap)));
  at::Tensor slots = at::empty({B * n}, fresh->options()), placed = at::empty({B}, fresh->options());
  const size_t need = plan_size(int(B), n);
  at::Tensor ws;
  if (need) ws = bytes_like(*bt, need);
  RUN("molt_plan_blocks",
      plan_entry(i32_out(*bt), i32_out(*have), i32(ctx), i32(fresh), i32_out(*pool), i32(shared), int(B), n,
                 int(bt->size(1)), int(cap), i32_out(slots), i32_out(placed), need ? ws.data_ptr() : nullptr, need,
                 stream));
  PyObject *a = THPVariable_Wrap(std::move(slots)), *b = THPVariable_Wrap(std::move(placed));
  PyObject* both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return both;
END_CALL

CALL(write, 7)  // k, v, k_cache, v_cache, slots, device, stream -> True
  const at::Tensor *k = in.tensor(), *v = in.tensor(), *kc = in.tensor(), *vc = in.tensor(), *slots = in.tensor();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  TAKE(in.fine && keys(*kc, dev) && values_of(*kc, *vc, dev));
  const int64_t nb = kc->size(0), H = kc->size(1), D = kc->size(3), T = slots->numel();
  int64_t ks, vs;
  TAKE(nb < (1l << 31) && H < (1l << 20) && T < (1l << 31) && ints(*slots, T, dev) &&
       rows(*k, kc->scalar_type(), T, H, D, dev, ks) && rows(*v, kc->scalar_type(), T, H, D, dev, vs));
  RUN("molt_kv_write",
      write_entry(k->const_data_ptr(), v->const_data_ptr(), ks, vs, i32(slots), int(T), int(H), int(D), int(nb),
                   code(kc->scalar_type()), kc->data_ptr(), vc->data_ptr(), stream));
  Py_RETURN_TRUE;
END_CALL

CALL(update, 8)  // k_cache, bounds, block_tables, starts, n, lens, device, stream -> True
  const at::Tensor *kc = in.tensor(), *bounds = in.tensor(), *bt = in.tensor(), *starts = in.tensor();
  const int n = in.number();
  const at::Tensor* lens = in.tensor_or_none();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  TAKE(in.fine && keys(*kc, dev) && bounds_of(*bounds, dev) && table(*bt, dev));
  const int64_t B = bt->size(0), nb = kc->size(0), H = kc->size(1), D = kc->size(3);
  TAKE(nb < (1l << 31) && H < (1l << 20) && bounds->size(0) == nb && bounds->size(1) == H &&
       bounds->size(2) == 2 * D + 16 && ints(*starts, B, dev) &&
       (!lens || ints(*lens, B, dev)));
  RUN("molt_key_bounds_update",
      update_entry(kc->const_data_ptr(), bounds->data_ptr(), i32(bt), i32(starts), i32(lens), int(B), n, int(H), int(D),
                    int(bt->size(1)), int(nb), code(kc->scalar_type()), stream));
  Py_RETURN_TRUE;
END_CALL

CALL(read, 4)  // bounds, ids, device, stream
  const at::Tensor *bounds = in.tensor(), *ids = in.tensor();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  TAKE(in.fine && bounds_of(*bounds, dev));
  const int64_t M = ids->numel(), nb = bounds->size(0), H = bounds->size(1), D = (bounds->size(2) - 16) / 2;
  TAKE(nb < (1l << 31) && H < (1l << 20) && M > 0 && M < (1l << 31) && ints(*ids, M, dev));
  RUN("molt_key_bounds_read", read_takes(int(M), int(H), int(D), int(nb)));
  const auto as = bounds->options().dtype(at::kFloat);
  at::Tensor hi = at::empty({M, H, D}, as), lo = at::empty({M, H, D}, as);
  RUN("molt_key_bounds_read",
      read_entry(bounds->const_data_ptr(), i32(ids), int(M), int(H), int(D), int(nb), static_cast<float*>(hi.data_ptr()),
                  static_cast<float*>(lo.data_ptr()), stream));
  PyObject *a = THPVariable_Wrap(std::move(hi)), *b = THPVariable_Wrap(std::move(lo));
  PyObject* both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return both;
END_CALL

CALL(select, 12)  // q, bounds, block_tables, context_lens, k, n_select, n_first, n_last, lens, workspace, device, stream
  const at::Tensor *q = in.tensor(), *bounds = in.tensor(), *bt = in.tensor(), *ctx = in.tensor();
  const int k = in.number(), N = in.number(), first = in.number(), last = in.number();
  const at::Tensor *lens = in.tensor_or_none(), *ws = in.tensor_or_none();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  void* room_at;
  size_t have;
  TAKE(in.fine && N > 0 && bounds_of(*bounds, dev) && table(*bt, dev) && floats(q->scalar_type()) &&
       whole(*q, q->scalar_type(), dev) && q->dim() == 3 && room(ws, dev, room_at, have));
  const int64_t B = bt->size(0), T = B * (int64_t(k) + 1), nb = bounds->size(0), H = bounds->size(1), Hq = q->size(1);
  const int64_t D = (bounds->size(2) - 16) / 2;
  TAKE(nb < (1l << 31) && H < (1l << 20) && Hq < (1l << 31) && q->size(0) == T && q->size(2) == D && ints(*ctx, B, dev) &&
       (!lens || ints(*lens, B, dev)));
  RUN("molt_select_blocks",
      select_takes(int(B), k, int(Hq), int(H), int(D), int(bt->size(1)), int(nb), N, first, last));
  at::Tensor out = at::empty({T, H, N}, bt->options());
  auto call = [&](void* at, size_t bytes) {
    return select_entry(q->const_data_ptr(), bounds->const_data_ptr(), i32(bt), i32(ctx), i32(lens), int(B), k, int(Hq),
                        int(H), int(D), int(bt->size(1)), int(nb), N, first, last, code(q->scalar_type()), i32_out(out), at,
                        bytes, stream);
  };
  int status = call(room_at, have);
  if (status == MOLT_ERR_WORKSPACE) {
    const at::Tensor own = bytes_like(*q, select_size(int(B), k, int(Hq), int(H), int(D), int(bt->size(1))));
    status = call(own.data_ptr(), own.nbytes());
  }
  RUN("molt_select_blocks", status);
  return THPVariable_Wrap(std::move(out));
END_CALL

CALL(attend, 10)  // q, k_cache, v_cache, block_tables, context_lens, k, blocks, workspace, device, stream
  const at::Tensor *q = in.tensor(), *kc = in.tensor(), *vc = in.tensor(), *bt = in.tensor(), *ctx = in.tensor();
  const int k = in.number();
  const at::Tensor *blocks = in.tensor(), *ws = in.tensor_or_none();
  const int dev = in.number();
  molt_stream_t stream = in.stream();
  void* room_at;
  size_t have;
  TAKE(in.fine && keys(*kc, dev) && values_of(*kc, *vc, dev) && table(*bt, dev) && whole(*q, kc->scalar_type(), dev) &&
       q->dim() == 3 && whole(*blocks, at::kInt, dev) && blocks->dim() == 3 && room(ws, dev, room_at, have));
  const int64_t B = bt->size(0), T = B * (int64_t(k) + 1), nb = kc->size(0), H = kc->size(1), D = kc->size(3);
  const int64_t Hq = q->size(1), N = blocks->size(2);
  TAKE(nb < (1l << 31) && H < (1l << 20) && Hq < (1l << 31) && N < (1l << 31) && q->size(0) == T && q->size(2) == D &&
       blocks->size(0) == T && blocks->size(1) == H && ints(*ctx, B, dev));
  RUN("molt_paged_attention_blocks",
      attend_takes(int(B), k, int(Hq), int(H), int(D), int(bt->size(1)), int(nb), int(N)));
  at::Tensor out = at::empty({T, Hq * D}, q->options());
  auto call = [&](void* at, size_t bytes) {
    return attend_entry(q->const_data_ptr(), kc->const_data_ptr(), vc->const_data_ptr(), i32(bt), i32(ctx), i32(blocks),
                        int(B), k, int(Hq), int(H), int(D), int(bt->size(1)), int(nb), int(N), code(kc->scalar_type()),
                        out.data_ptr(), at, bytes, stream);
  };
  int status = call(room_at, have);
  if (status == MOLT_ERR_WORKSPACE) {
    const at::Tensor own = bytes_like(*q, attend_size(int(B), k, int(Hq), int(H), int(D), int(N)));
    status = call(own.data_ptr(), own.nbytes());
  }
  RUN("molt_paged_attention_blocks", status);
  return THPVariable_Wrap(std::move(out));
END_CALL

// MoltError, then the addresses of the entries
PyObject* set_entries(PyObject*, PyObject* args) {
  PyObject* error;
  unsigned long long a[14];
  if (!PyArg_ParseTuple(args, "OKKKKKKKKKKKKKK", &error, a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8, a + 9,
                        a + 10, a + 11, a + 12, a + 13))
    return nullptr;
  Py_INCREF(error);
  Py_XDECREF(error_class);
  error_class = error;
  last_error = reinterpret_cast<decltype(last_error)>(a[0]);
  plan_entry = reinterpret_cast<decltype(plan_entry)>(a[1]);
  plan_size = reinterpret_cast<decltype(plan_size)>(a[2]);
  write_entry = reinterpret_cast<decltype(write_entry)>(a[3]);
  update_entry = reinterpret_cast<decltype(update_entry)>(a[4]);
  read_entry = reinterpret_cast<decltype(read_entry)>(a[5]);
  select_entry = reinterpret_cast<decltype(select_entry)>(a[6]);
  select_size = reinterpret_cast<decltype(select_size)>(a[7]);
  attend_entry = reinterpret_cast<decltype(attend_entry)>(a[8]);
  attend_size = reinterpret_cast<decltype(attend_size)>(a[9]);
  plan_takes = reinterpret_cast<decltype(plan_takes)>(a[10]);
  read_takes = reinterpret_cast<decltype(read_takes)>(a[11]);
  select_takes = reinterpret_cast<decltype(select_takes)>(a[12]);
  attend_takes = reinterpret_cast<decltype(attend_takes)>(a[13]);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(plan), FAST(write), FAST(update), FAST(read), FAST(select), FAST(attend),
                         {"set_entries", set_entries, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
