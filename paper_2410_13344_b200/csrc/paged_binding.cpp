// The paged-cache calls of the Python binding, natively: arguments checked, outputs allocated, the C ABI called on the tensors' device and its
// current stream.  A decoding step makes several of these calls a layer, each of a few microseconds of GPU time; by way of Python's
// attributes and ctypes a call of kv_append took 8.9 us of host time, one of paged_attention 15 and one of page_select 20.
//
// The functions of libcerb.so come from binding.py (setup), which has the library loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "cerb.h"

namespace {

struct Library {
  decltype(&cerb_pages_plan) pages_plan;
  decltype(&cerb_pages_trim) pages_trim;
  decltype(&cerb_kv_append) kv_append;
  decltype(&cerb_paged_attention_scratch_bytes) attention_scratch;
  decltype(&cerb_paged_attention) attention;
  decltype(&cerb_page_select_scratch_bytes) select_scratch;
  decltype(&cerb_page_select) select;
} lib;
PyObject* error_class = nullptr;         // binding.CerbError(code, what)
PyObject* plan_class = nullptr;          // binding.PagePlan

// What a refusal is thrown as, on its way to Python.
struct Refused {
  int code;
  const char* what;
  const char* why;
};
[[noreturn]] void refuse(const char* what, const char* why, int code = CERB_E_ARG) { throw Refused{code, what, why}; }

PyObject* raise(const Refused& r) {
  PyObject* e = r.why ? PyObject_CallFunction(error_class, "iN", r.code, PyUnicode_FromFormat("%s (%s)", r.what, r.why))
                      : PyObject_CallFunction(error_class, "is", r.code, r.what);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  return nullptr;
}

void done(int rc, const char* what) {
  if (rc != CERB_OK) throw Refused{rc, what, nullptr};
}

// ---- arguments ----
const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(what, "an argument is not a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* what) { return o == Py_None ? nullptr : &tensor(o, what); }
int32_t whole(PyObject* o, const char* what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  if (v < INT_MIN || v > INT_MAX) refuse(what, "a number is out of range");
  return (int32_t)v;
}

int device_of(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) refuse(what, "tensors must be on a GPU");
  return t.get_device();
}
// Lengths, tables, lists and counts: int32, in one piece, on that GPU.
int32_t* index_data(const at::Tensor& t, int device, const char* what) {
  if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse(what, "lengths, tables, lists and counts are contiguous int32 tensors");
  if (!t.is_cuda() || t.get_device() != device) refuse(what, "tensors are on different devices");
  return (int32_t*)t.data_ptr();
}
int dtype_of(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kBFloat16) return CERB_BF16;
  if (t.scalar_type() == at::kFloat) return CERB_F32;
  refuse(what, "bfloat16 or float32");
}
int32_t size32(int64_t n, const char* what) {
  if (n > INT_MAX) refuse(what, "a dimension is out of range", CERB_E_SHAPE);
  return (int32_t)n;
}
// Two tensors of a cache: alike, contiguous, on the device.
void alike(const at::Tensor& a, const at::Tensor& b, int dims, int device, const char* what, const char* why) {
  if (a.dim() != dims || !a.sizes().equals(b.sizes()) || a.scalar_type() != b.scalar_type() || !a.is_contiguous() || !b.is_contiguous()) refuse(what, why);
  if (!a.is_cuda() || !b.is_cuda() || a.get_device() != device || b.get_device() != device) refuse(what, "tensors are on different devices");
}
const char* const kPools = "pools are [pages][KV heads][16][head_dim], alike and contiguous";
const char* const kSummaries = "k_min and k_max are [pages][KV heads][head_dim], alike and contiguous";

// A [rows][heads][head_dim] operand, strided, of the cache's type.
void* operand(const at::Tensor& t, int64_t rows, int64_t heads, int64_t dh, const at::Tensor& like, int device, int64_t* row, int64_t* head, const char* what,
              const char* why) {
  if (t.dim() != 3 || t.size(0) != rows || t.size(1) != heads || t.size(2) != dh || t.scalar_type() != like.scalar_type() || t.stride(2) != 1) refuse(what, why);
  if (!t.is_cuda() || t.get_device() != device) refuse(what, "tensors are on different devices");
  *row = rows > 1 ? t.stride(0) : 0;               // (torch leaves any stride where there is nothing to step over)
  *head = heads > 1 ? t.stride(1) : 0;
  return t.data_ptr();
}

at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, int device) {
  return at::detail::empty_cuda(sizes, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}
// Results of a call are parts of one piece of memory, each on 16 bytes: an allocation is a microsecond.
struct Parts {
  at::Tensor all;
  int64_t used = 0;
  static int64_t bytes(at::IntArrayRef sizes, at::ScalarType type) {
    return (c10::multiply_integers(sizes) * (int64_t)c10::elementSize(type) + 15) / 16 * 16;
  }
  Parts(int64_t bytes, int device) : all(make({bytes}, at::kByte, device)) {}
  at::Tensor next(at::IntArrayRef sizes, at::ScalarType type) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(type));
    impl->set_storage_offset(used / (int64_t)c10::elementSize(type));
    impl->set_sizes_contiguous(sizes);
    used += bytes(sizes, type);
    return at::Tensor(std::move(impl));
  }
};
void* stream_of(int device) { return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

// Runs a call with the tensors' device current, and turns what is thrown into a Python error.
template <typename F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    at::AutoDispatchBelowADInplaceOrView no_grad;
    return f();
  } catch (const Refused& r) {
    return raise(r);
  }
  END_HANDLE_TH_ERRORS
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
  return false;
}

// ---- the calls ----
cerb_pages book(PyObject* const* a, const at::Tensor& n, int device, const char* what) {          // lens, page_table, free_pages, n_free
  const at::Tensor &lens = tensor(a[0], what), &table = tensor(a[1], what), &free = tensor(a[2], what), &n_free = tensor(a[3], what);
  cerb_pages s;
  s.len = index_data(lens, device, what);
  s.page_table = index_data(table, device, what);
  s.free_pages = index_data(free, device, what);
  s.n_free = index_data(n_free, device, what);
  const int64_t B = lens.numel();
  if (lens.dim() != 1 || n.dim() != 1 || n.size(0) != B || table.dim() != 2 || table.size(0) != B || table.size(1) < 1 || free.dim() != 1 || n_free.numel() != 1)
    refuse(what, "lens [B], a number a request, page_table [B][one column at least], free_pages [capacity], n_free [1]");
  s.B = size32(B, what);
  s.max_pages = size32(table.size(1), what);
  s.free_cap = size32(free.numel(), what);
  return s;
}

PyObject* pages_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {       // n_new, lens, page_table, free_pages, n_free, rows
  if (!count(n, 6)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* what = "cerb_pages_plan";
    const at::Tensor& n_new = tensor(a[0], what);
    const int device = device_of(n_new, what);
    const int32_t* want = index_data(n_new, device, what);
    const cerb_pages s = book(a + 1, n_new, device, what);
    const int32_t rows = whole(a[5], what);
    if (rows < 0) refuse(what, "rows is negative");
    if (s.B > 8192 || rows > 1 << 30) refuse(what, "more than 8192 requests or 2^30 rows", CERB_E_SHAPE);        // (ahead of the allocations)
    const c10::cuda::OptionalCUDAGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)device));
    const int64_t sizes[5] = {rows, rows, rows, s.B + 1, s.B};
    int64_t bytes = 0;
    for (const int64_t n : sizes) bytes += Parts::bytes({n}, at::kInt);
    Parts parts(bytes, device);
    at::Tensor out[5];
    int32_t* p[5];
    for (int i = 0; i < 5; ++i) {
      out[i] = parts.next({sizes[i]}, at::kInt);
      p[i] = (int32_t*)out[i].data_ptr();
    }
    done(lib.pages_plan(&s, want, rows, p[0], p[1], p[2], p[3], p[4], stream_of(device)), what);
    return PyObject_CallFunction(plan_class, "NNNNN", THPVariable_Wrap(out[0]), THPVariable_Wrap(out[1]), THPVariable_Wrap(out[2]), THPVariable_Wrap(out[3]),
                                 THPVariable_Wrap(out[4]));
  });
}

PyObject* pages_trim(PyObject*, PyObject* const* a, Py_ssize_t n) {       // keep, lens, page_table, free_pages, n_free
  if (!count(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* what = "cerb_pages_trim";
    const at::Tensor& keep = tensor(a[0], what);
    const int device = device_of(keep, what);
    const int32_t* want = index_data(keep, device, what);
    const cerb_pages s = book(a + 1, keep, device, what);
    const c10::cuda::OptionalCUDAGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)device));
    done(lib.pages_trim(&s, want, stream_of(device)), what);
    Py_RETURN_NONE;
  });
}

PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {        // k, v, slot, k_pool, v_pool, k_min, k_max
  if (!count(n, 7)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* what = "cerb_kv_append";
    const at::Tensor &k = tensor(a[0], what), &v = tensor(a[1], what), &slot = tensor(a[2], what), &k_pool = tensor(a[3], what), &v_pool = tensor(a[4], what);
    const at::Tensor *k_min = maybe(a[5], what), *k_max = maybe(a[6], what);
    const int device = device_of(k_pool, what);
    alike(k_pool, v_pool, 4, device, what, kPools);
    if (k_pool.size(2) != CERB_PAGE) refuse(what, kPools);
    cerb_kv_append_args g;
    g.dtype = dtype_of(k_pool, what);
    g.slot = index_data(slot, device, what);
    g.T = size32(slot.numel(), what);
    g.n_pool_pages = size32(k_pool.size(0), what);
    g.n_kv_heads = size32(k_pool.size(1), what);
    g.head_dim = size32(k_pool.size(3), what);
    g.k = operand(k, g.T, g.n_kv_heads, g.head_dim, k_pool, device, &g.k_row_stride, &g.k_head_stride, what,
                  "k is [slots][KV heads][head_dim], of the pools' type, the elements of a head next to one another");
    g.v = operand(v, g.T, g.n_kv_heads, g.head_dim, k_pool, device, &g.v_row_stride, &g.v_head_stride, what,
                  "v is [slots][KV heads][head_dim], of the pools' type, the elements of a head next to one another");
    g.k_pool = k_pool.data_ptr();
    g.v_pool = v_pool.data_ptr();
    g.k_min = g.k_max = nullptr;
    if (!k_min != !k_max) refuse(what, "k_min and k_max come together");
    if (k_min) {
      alike(*k_min, *k_max, 3, device, what, kSummaries);
      if (k_min->scalar_type() != k_pool.scalar_type() || k_min->size(0) != k_pool.size(0) || k_min->size(1) != k_pool.size(1) || k_min->size(2) != k_pool.size(3))
        refuse(what, "k_min and k_max are of other pages than the pools, or of another type");
      g.k_min = k_min->data_ptr();
      g.k_max = k_max->data_ptr();
    }
    const c10::cuda::OptionalCUDAGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)device));
    done(lib.kv_append(&g, stream_of(device)), what);
    Py_RETURN_NONE;
  });
}

struct Queries {
  int32_t B, H, max_pages;
  const void* q;
  int64_t row, head;
  const int32_t *table, *len;
};
Queries queries(const at::Tensor& q, const at::Tensor& table, const at::Tensor& lens, int64_t Hk, int64_t dh, const at::Tensor& like, int device,
                const char* what) {
  Queries r;
  if (q.dim() != 3 || Hk < 1 || q.size(1) < 1 || q.size(1) % Hk) refuse(what, "q is [B][heads][head_dim], its heads a multiple of the KV heads");
  r.B = size32(q.size(0), what);
  r.H = size32(q.size(1), what);
  if (table.dim() != 2 || table.size(0) != r.B || table.size(1) < 1 || lens.dim() != 1 || lens.size(0) != r.B)
    refuse(what, "a length and a row of the page table for every sequence");
  r.max_pages = size32(table.size(1), what);
  r.table = index_data(table, device, what);
  r.len = index_data(lens, device, what);
  r.q = operand(q, r.B, r.H, dh, like, device, &r.row, &r.head, what, "q is [B][heads][head_dim], of the cache's type, the elements of a head next to one another");
  return r;
}
// The scratch that was given, or one of this many bytes.
at::Tensor scratch_of(const at::Tensor* given, size_t need, int device, const char* what) {
  if (!given) return need ? make({(int64_t)need}, at::kByte, device) : at::Tensor();
  if (!given->is_cuda() || given->get_device() != device || given->scalar_type() != at::kByte || !given->is_contiguous())
    refuse(what, "scratch is a contiguous uint8 tensor on the same device");
  return *given;
}

// q, k_min, k_max, page_table, lens, n_pages, max_len, n_first, n_last, scratch
PyObject* page_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 10)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* what = "cerb_page_select";
    const at::Tensor &q = tensor(a[0], what), &k_min = tensor(a[1], what), &k_max = tensor(a[2], what), &table = tensor(a[3], what), &lens = tensor(a[4], what);
    const int device = device_of(k_min, what);
    alike(k_min, k_max, 3, device, what, kSummaries);
    cerb_page_select_args g;
    g.dtype = dtype_of(k_min, what);
    const Queries r = queries(q, table, lens, k_min.size(1), k_min.size(2), k_min, device, what);
    g.B = r.B;
    g.n_heads = r.H;
    g.n_kv_heads = size32(k_min.size(1), what);
    g.head_dim = size32(k_min.size(2), what);
    g.max_pages = r.max_pages;
    g.n_pool_pages = size32(k_min.size(0), what);
    g.q = r.q;
    g.q_row_stride = r.row;
    g.q_head_stride = r.head;
    g.k_min = k_min.data_ptr();
    g.k_max = k_max.data_ptr();
    g.page_table = r.table;
    g.len = r.len;
    g.max_sel = whole(a[5], what);
    g.max_len = whole(a[6], what);
    g.n_first = whole(a[7], what);
    g.n_last = whole(a[8], what);
    if (g.max_sel < 1 || g.n_first < 0 || g.n_last < 0 || g.max_len < 1) refuse(what, "counts are not negative, n_pages and max_len one at least");
    size_t need = 0;
    done(lib.select_scratch(g.dtype, g.B, g.n_heads, g.n_kv_heads, g.head_dim, g.max_pages, g.max_len, &need), what);
    const c10::cuda::OptionalCUDAGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)device));
    const at::Tensor scratch = scratch_of(maybe(a[9], what), need, device, what);
    g.scratch = scratch.defined() ? scratch.data_ptr() : nullptr;
    g.scratch_bytes = scratch.defined() ? (size_t)scratch.numel() : 0;
    const int64_t lists[3] = {g.B, g.n_kv_heads, g.max_sel}, counts[1] = {g.B};
    Parts parts(Parts::bytes(lists, at::kInt) + Parts::bytes(counts, at::kInt), device);
    const at::Tensor sel = parts.next(lists, at::kInt), n_sel = parts.next(counts, at::kInt);
    g.sel = (int32_t*)sel.data_ptr();
    g.n_sel = (int32_t*)n_sel.data_ptr();
    done(lib.select(&g, stream_of(device)), what);
    return Py_BuildValue("NN", THPVariable_Wrap(sel), THPVariable_Wrap(n_sel));
  });
}

// q, k_pool, v_pool, page_table, lens, scale, max_len, window, sel, n_sel, want_lse, scratch
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  return guarded([&]() -> PyObject* {
    const char* what = "cerb_paged_attention";
    const at::Tensor &q = tensor(a[0], what), &k_pool = tensor(a[1], what), &v_pool = tensor(a[2], what), &table = tensor(a[3], what), &lens = tensor(a[4], what);
    const at::Tensor *sel = maybe(a[8], what), *n_sel = maybe(a[9], what);
    const int device = device_of(k_pool, what);
    alike(k_pool, v_pool, 4, device, what, kPools);
    if (k_pool.size(2) != CERB_PAGE) refuse(what, kPools);
    cerb_paged_attn_args g;
    g.dtype = dtype_of(k_pool, what);
    const Queries r = queries(q, table, lens, k_pool.size(1), k_pool.size(3), k_pool, device, what);
    g.B = r.B;
    g.n_heads = r.H;
    g.n_kv_heads = size32(k_pool.size(1), what);
    g.head_dim = size32(k_pool.size(3), what);
    g.max_pages = r.max_pages;
    g.n_pool_pages = size32(k_pool.size(0), what);
    g.q = r.q;
    g.q_row_stride = r.row;
    g.q_head_stride = r.head;
    g.k_pool = k_pool.data_ptr();
    g.v_pool = v_pool.data_ptr();
    g.page_table = r.table;
    g.len = r.len;
    g.scale = (float)PyFloat_AsDouble(a[5]);
    if (g.scale == -1.f && PyErr_Occurred()) throw python_error();
    g.max_len = whole(a[6], what);
    g.window = whole(a[7], what);
    if (g.max_len < 1 || g.window < 0) refuse(what, "max_len is one at least, window not negative");
    g.sel = g.n_sel = nullptr;
    g.max_sel = 0;
    if (!sel != !n_sel) refuse(what, "sel and n_sel come together");
    if (sel) {
      g.sel = index_data(*sel, device, what);
      g.n_sel = index_data(*n_sel, device, what);
      if (sel->dim() != 3 || sel->size(0) != g.B || sel->size(1) != g.n_kv_heads || sel->size(2) < 1 || n_sel->dim() != 1 || n_sel->size(0) != g.B)
        refuse(what, "sel is [B][KV heads][pages], n_sel [B]");
      g.max_sel = size32(sel->size(2), what);
    }
    const int lse_wanted = PyObject_IsTrue(a[10]);
    if (lse_wanted < 0) throw python_error();
    size_t need = 0;
    done(lib.attention_scratch(g.dtype, g.B, g.n_heads, g.n_kv_heads, g.head_dim, g.max_len, g.window, g.max_sel, &need), what);
    const c10::cuda::OptionalCUDAGuard on(c10::Device(c10::kCUDA, (c10::DeviceIndex)device));
    const at::Tensor scratch = scratch_of(maybe(a[11], what), need, device, what);
    g.scratch = scratch.defined() ? scratch.data_ptr() : nullptr;
    g.scratch_bytes = scratch.defined() ? (size_t)scratch.numel() : 0;
    const int64_t outs[3] = {g.B, g.n_heads, g.head_dim};
    Parts parts(Parts::bytes(outs, q.scalar_type()) + (lse_wanted ? Parts::bytes({g.B, g.n_heads}, at::kFloat) : 0), device);
    const at::Tensor out = parts.next(outs, q.scalar_type());
    at::Tensor lse;
    if (lse_wanted) lse = parts.next({g.B, g.n_heads}, at::kFloat);
    g.out = out.data_ptr();
    g.lse = lse_wanted ? (float*)lse.data_ptr() : nullptr;
    done(lib.attention(&g, stream_of(device)), what);
    if (!lse_wanted) return Py_BuildValue("NO", THPVariable_Wrap(out), Py_None);
    return Py_BuildValue("NN", THPVariable_Wrap(out), THPVariable_Wrap(lse));
  });
}

// error class, plan class, addresses of the library's functions in the order of Library
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  void* at[sizeof(Library) / sizeof(void*)];
  for (size_t i = 0; i < sizeof(at) / sizeof(*at); ++i) {
    PyObject* item = PySequence_GetItem(a[2], (Py_ssize_t)i);
    if (!item) return nullptr;
    at[i] = PyLong_AsVoidPtr(item);
    Py_DECREF(item);
    if (!at[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a function without an address");
      return nullptr;
    }
  }
  memcpy(&lib, at, sizeof(at));
  Py_INCREF(a[0]);
  Py_XSETREF(error_class, a[0]);
  Py_INCREF(a[1]);
  Py_XSETREF(plan_class, a[1]);
  Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(setup),     METHOD(pages_plan),  METHOD(pages_trim),      METHOD(kv_append),
                         METHOD(page_select), METHOD(paged_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() { return PyModule_Create(&module); }
