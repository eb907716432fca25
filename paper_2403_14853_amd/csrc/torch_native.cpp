// Native half of the Python binding (CPython module _isp_torch): argument marshalling between torch tensors and
// the C ABI (include/isp.h), and the autograd nodes.  No arithmetic here.
//
// Why it is not Python: on small graphs a call costs more on the host than on the GPU.  Marshalled through ctypes a
// SpMM of 4,096 rows took 8.8 us of host time for 5 us of kernel, and a forward + backward through a Python
// autograd.Function 48 - 115 us: the engine runs the backward on a thread of its own, and every Python statement
// there competes for the interpreter.  Measured after the move: see the comments at spmm() and at the nodes.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/utils/pybind.h>
#include <ATen/ATen.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <hip/hip_runtime_api.h>
#include <algorithm>
#include <atomic>
#include <cmath>
#include <memory>
#include <mutex>
#include <vector>
#include "isp.h"

namespace {

using at::Tensor;
using torch::autograd::variable_list;

PyObject* g_check = nullptr;      // binding._check: raises IspError for a status
PyObject* g_transpose = nullptr;  // binding.csr_transpose_cached

// The stream of a call.  own: one of torch's, which live as long as the process; a stream that somebody else made may be gone when
// a handle is dropped.
struct Where {
  void* s;
  bool own;
};

// A handle as the Python object CSR owns it; destroy() on that object clears h for everybody who shares the cell.
struct Cell {
  std::atomic<isp_csr_t*> h{nullptr};
  int64_t n_rows = 0, n_cols = 0, nnz = 0;

  // The streams that calls on the handle have been put on.
  struct Use {
    void* s;
    int device;
  };
  void ran_on(Where w) {
    if (!w.own) {
      foreign.store(true, std::memory_order_relaxed);
      return;
    }
    if (w.s == last.load(std::memory_order_relaxed)) return;
    std::lock_guard<std::mutex> lock(m);
    last.store(w.s, std::memory_order_relaxed);
    for (const Use& u : uses)
      if (u.s == w.s) return;
    hipDevice_t device = 0;
    if (w.s ? hipStreamGetDevice((hipStream_t)w.s, &device) != hipSuccess : hipGetDevice(&device) != hipSuccess) {
      foreign.store(true, std::memory_order_relaxed);
      return;
    }
    uses.push_back({w.s, device});
  }
  std::atomic<bool> foreign{false};  // a call ran on a stream that is not one of torch's
  std::mutex m;
  std::vector<Use> uses;

 private:
  static inline char none;  // (the default stream is a null pointer)
  std::atomic<void*> last{&none};
};
using CellPtr = std::shared_ptr<Cell>;

// What autograd.SparseGraph keeps on this side.
struct Graph {
  CellPtr A, At;          // At: the cached transpose, once it has been built
  Tensor values;          // undefined when all entries are 1
  uint32_t version = 0;   // of `values` when the handle last read them
  PyObject* csr = nullptr;  // the CSR object (keeps the handle and every tensor it borrows alive)
  ~Graph() {
    if (csr && Py_IsInitialized()) {
      pybind11::gil_scoped_acquire gil;  // (an autograd node may be the last owner, on a thread of the engine)
      Py_DECREF(csr);
    }
  }
};
using GraphPtr = std::shared_ptr<Graph>;

const char* const CELL = "isp.cell";
const char* const GRAPH = "isp.graph";

template <class T>
void drop(PyObject* c) {
  delete static_cast<std::shared_ptr<T>*>(PyCapsule_GetPointer(c, PyCapsule_GetName(c)));
}
template <class T>
PyObject* wrap(std::shared_ptr<T> p, const char* name) {
  auto* box = new std::shared_ptr<T>(std::move(p));
  PyObject* c = PyCapsule_New(box, name, drop<T>);
  if (!c) delete box;
  return c;
}
Cell* cell_of(PyObject* c) {
  auto* p = static_cast<CellPtr*>(PyCapsule_GetPointer(c, CELL));
  return p ? p->get() : nullptr;
}

PyObject* fail(const char* what) {
  PyErr_SetString(PyExc_AssertionError, what);
  return nullptr;
}

// One dense operand: fp32 rows on the GPU, contiguous within a row.
struct Dense {
  float* p;
  int64_t rows, d, ld;
};
const char* dense_of(const Tensor& t, Dense& o) {
  if (t.dim() != 2) return "a dense operand has two dimensions";
  if (!t.is_cuda()) return "a dense operand lives on the GPU";
  if (t.scalar_type() != at::kFloat) return "a dense operand is float32";
  if (t.stride(1) != 1) return "the rows of a dense operand are contiguous";
  o.p = static_cast<float*>(t.data_ptr());
  o.rows = t.size(0);
  o.d = t.size(1);
  o.ld = o.rows > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), o.d);
  return nullptr;
}
// (THPVariable_Unpack trusts its argument: whatever comes from a caller is looked at first)
bool is_tensor(PyObject* o) {
  if (THPVariable_Check(o)) return true;
  PyErr_SetString(PyExc_TypeError, "a torch tensor is expected");
  return false;
}
bool dense_of(PyObject* o, Dense& out) {
  if (!is_tensor(o)) return false;
  const char* bad = dense_of(THPVariable_Unpack(o), out);
  if (bad) fail(bad);
  return !bad;
}

Where here() {  // the current stream of the current device
  const auto s = c10::hip::getCurrentHIPStream();
  void* const p = s.stream();
  return {p, !p || s.id() != reinterpret_cast<intptr_t>(p)};  // (the id of a stream that torch has not made is its address)
}
Where stream_of(PyObject* o) {  // None: the current one; else its address, negative if it is not one of torch's
  if (o == Py_None) return here();
  const long long p = PyLong_AsLongLong(o);
  return {reinterpret_cast<void*>(p < 0 ? -p : p), p >= 0};
}

#define ISP_ARGS(n)                                                                            \
  if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }

template <class F>
PyObject* call(Cell* c, Where w, F&& f) {  // the library call on c's handle with the interpreter released, its status as a Python int
  isp_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f(c->h.load(), w.s);
  if (st == ISP_OK || st == ISP_EHIP) c->ran_on(w);  // (else nothing has been launched)
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// (h as a ctypes integer, n_rows, n_cols, nnz) -> cell
PyObject* py_cell(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(4)
  auto c = std::make_shared<Cell>();
  c->h = static_cast<isp_csr_t*>(PyLong_AsVoidPtr(a[0]));
  c->n_rows = PyLong_AsLongLong(a[1]);
  c->n_cols = PyLong_AsLongLong(a[2]);
  c->nnz = PyLong_AsLongLong(a[3]);
  if (PyErr_Occurred()) return nullptr;
  return wrap(std::move(c), CELL);
}
// (cell, stream): a call through ctypes on that stream has used the handle
PyObject* py_cell_ran(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(2)
  Cell* c = cell_of(a[0]);
  if (!c) return nullptr;
  const Where w = stream_of(a[1]);
  if (PyErr_Occurred()) return nullptr;
  c->ran_on(w);
  Py_RETURN_NONE;
}
// (cell) -> has a call run on a stream that is not one of torch's?
PyObject* py_cell_foreign(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(1)
  Cell* c = cell_of(a[0]);
  if (!c) return nullptr;
  return PyBool_FromLong(c->foreign.load());
}
// (cells, list, cell or None): before the list's tensors are let go.  The allocator hears of every stream that calls on the cells' handles
// ran on, and reuses the memory once those are through; the other cell (an alias's source, whose arrays the calls read) takes the
// streams over.
PyObject* py_cells_release(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(3)
  Cell* heir = nullptr;
  if (a[2] != Py_None && !(heir = cell_of(a[2]))) return nullptr;
  if (!PyList_Check(a[0]) || !PyList_Check(a[1])) return fail("lists of cells and of what they borrow");
  std::vector<Cell::Use> uses;
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[0]); ++i) {
    Cell* c = cell_of(PyList_GET_ITEM(a[0], i));
    if (!c) return nullptr;
    std::lock_guard<std::mutex> lock(c->m);
    uses.insert(uses.end(), c->uses.begin(), c->uses.end());
    if (heir && c->foreign.load()) heir->foreign.store(true);
  }
  for (size_t u = 0; u < uses.size(); ++u) {
    bool again = false;
    for (size_t v = 0; v < u; ++v) again |= uses[v].s == uses[u].s;
    if (again) continue;
    if (heir) heir->ran_on({uses[u].s, true});
    const auto dev = static_cast<c10::DeviceIndex>(uses[u].device);
    const auto s = uses[u].s ? c10::hip::getStreamFromExternal((hipStream_t)uses[u].s, dev) : c10::hip::getDefaultHIPStream(dev);
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[1]); ++i) {
      PyObject* o = PyList_GET_ITEM(a[1], i);
      // (Tensor.record_stream without the dispatcher: a mode that is active where a handle happens to go has no part in this)
      if (THPVariable_Check(o)) c10::hip::HIPCachingAllocator::recordStream(THPVariable_Unpack(o).storage().data_ptr(), s);
    }
  }
  Py_RETURN_NONE;
}
PyObject* py_cell_clear(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(1)
  Cell* c = cell_of(a[0]);
  if (!c) return nullptr;
  c->h = nullptr;
  Py_RETURN_NONE;
}

// (cell, X, Y, stream): a 4,096-row call 8.8 -> 3.3 us of host time (most of it the kernel launch)
template <isp_status (*FN)(const isp_csr_t*, const float*, int64_t, int32_t, float*, int64_t, void*)>
PyObject* py_spmm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(4)
  Cell* c = cell_of(a[0]);
  Dense X, Y;
  if (!c || !dense_of(a[1], X) || !dense_of(a[2], Y)) return nullptr;
  if (X.rows != c->n_cols || Y.rows != c->n_rows || Y.d != X.d) return fail("X has A's columns as rows, Y its rows, both the same width");
  const Where w = stream_of(a[3]);
  if (PyErr_Occurred()) return nullptr;
  return call(c, w, [&](isp_csr_t* h, void* s) { return FN(h, X.p, X.ld, (int32_t)X.d, Y.p, Y.ld, s); });
}

// (cell, U, V, out, flags, stream)
PyObject* py_sddmm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(6)
  Cell* c = cell_of(a[0]);
  Dense U, V;
  if (!c || !dense_of(a[1], U) || !dense_of(a[2], V)) return nullptr;
  if (!THPVariable_Check(a[3])) return fail("out is a tensor");
  const Tensor& out = THPVariable_Unpack(a[3]);
  if (U.rows != c->n_rows || V.rows != c->n_cols || V.d != U.d || out.numel() != c->nnz) return fail("U has A's rows, V its columns as rows, out one value per entry");
  const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[4]);
  const Where w = stream_of(a[5]);
  if (PyErr_Occurred()) return nullptr;
  float* o = static_cast<float*>(out.data_ptr());
  return call(c, w, [&](isp_csr_t* h, void* s) { return isp_sddmm(h, U.p, U.ld, V.p, V.ld, (int32_t)U.d, flags, o, s); });
}

// (cell, X, Y, op, stream)
PyObject* py_fusedmm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(5)
  Cell* c = cell_of(a[0]);
  Dense X, Y;
  if (!c || !dense_of(a[1], X) || !dense_of(a[2], Y)) return nullptr;
  if (X.rows != c->n_rows || Y.rows != X.rows || Y.d != X.d) return fail("X and Y have A's rows and one width");
  const int op = (int)PyLong_AsLong(a[3]);
  const Where w = stream_of(a[4]);
  if (PyErr_Occurred()) return nullptr;
  return call(c, w, [&](isp_csr_t* h, void* s) { return isp_fusedmm(h, X.p, X.ld, (int32_t)X.d, op, Y.p, Y.ld, s); });
}

// (cell, X, dY, dX, op, stream)
PyObject* py_fusedmm_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(6)
  Cell* c = cell_of(a[0]);
  Dense X, G, O;
  if (!c || !dense_of(a[1], X) || !dense_of(a[2], G) || !dense_of(a[3], O)) return nullptr;
  if (G.rows != X.rows || G.d != X.d || O.rows != X.rows || O.d != X.d) return fail("X, dY and dX have one shape");
  const int op = (int)PyLong_AsLong(a[4]);
  const Where w = stream_of(a[5]);
  if (PyErr_Occurred()) return nullptr;
  return call(c, w, [&](isp_csr_t* h, void* s) { return isp_fusedmm_backward(h, X.p, X.ld, G.p, G.ld, (int32_t)X.d, op, O.p, O.ld, s); });
}

// The arg array of min / max (None: absent).
bool arg_of(PyObject* o, const Cell* c, int64_t d, bool check, int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  if (!THPVariable_Check(o)) { fail("arg is a tensor"); return false; }
  const Tensor& t = THPVariable_Unpack(o);
  if (check && (t.scalar_type() != at::kInt || !t.is_contiguous() || t.dim() != 2 || t.size(0) != c->n_rows || t.size(1) != d)) {
    fail("arg is int32, contiguous, one row per row of A");
    return false;
  }
  *out = static_cast<int32_t*>(t.data_ptr());
  return true;
}

// (cell, X, Y, reduce, arg, stream)
PyObject* py_spmm_reduce(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(6)
  Cell* c = cell_of(a[0]);
  Dense X, Y;
  int32_t* arg;
  if (!c || !dense_of(a[1], X) || !dense_of(a[2], Y)) return nullptr;
  if (X.rows != c->n_cols || Y.rows != c->n_rows || Y.d != X.d) return fail("X has A's columns as rows, Y its rows, both the same width");
  if (!arg_of(a[4], c, X.d, true, &arg)) return nullptr;
  const int red = (int)PyLong_AsLong(a[3]);
  const Where w = stream_of(a[5]);
  if (PyErr_Occurred()) return nullptr;
  return call(c, w, [&](isp_csr_t* h, void* s) { return isp_spmm_reduce(h, X.p, X.ld, (int32_t)X.d, red, Y.p, Y.ld, arg, s); });
}

// (cell, dY, dX, reduce, arg, stream)
PyObject* py_spmm_reduce_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(6)
  Cell* c = cell_of(a[0]);
  Dense G, O;
  int32_t* arg;
  if (!c || !dense_of(a[1], G) || !dense_of(a[2], O)) return nullptr;
  if (G.rows != c->n_rows || O.rows != c->n_cols || O.d != G.d) return fail("dY has A's rows, dX its columns as rows, both the same width");
  if (!arg_of(a[4], c, G.d, false, &arg)) return nullptr;
  const int red = (int)PyLong_AsLong(a[3]);
  const Where w = stream_of(a[5]);
  if (PyErr_Occurred()) return nullptr;
  return call(c, w, [&](isp_csr_t* h, void* s) { return isp_spmm_reduce_backward(h, G.p, G.ld, (int32_t)G.d, red, arg, O.p, O.ld, s); });
}

// ---- operands of the operators that take half precision too ----------------------------------------------------------
// Rows on the current device, fp32 or 16 bits, contiguous within a row.
struct Mat {
  void* p;
  int64_t rows, d, ld;
  int type;
};
int type_of(at::ScalarType t) { return t == at::kFloat ? ISP_F32 : t == at::kBFloat16 ? ISP_BF16 : t == at::kHalf ? ISP_F16 : -1; }
bool is_here(const Tensor& t) { return t.is_cuda() && t.device().index() == c10::hip::current_device(); }
const char* mat_of(const Tensor& t, Mat& o) {
  if (t.dim() != 2) return "a dense operand has two dimensions";
  if (!is_here(t)) return "a dense operand lives on the current GPU";
  o.type = type_of(t.scalar_type());
  if (o.type < 0) return "a dense operand is float32, bfloat16 or float16";
  if (t.stride(1) != 1 && t.size(1) > 1) return "the rows of a dense operand are contiguous";
  o.p = t.data_ptr();
  o.rows = t.size(0);
  o.d = t.size(1);
  if (o.d > INT32_MAX) return "a dense operand has rows of at most 2^31 - 1 elements";
  o.ld = o.rows > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), o.d);
  return nullptr;
}
// A dense array of so many elements of one type (undefined: absent).
const char* array_of(const Tensor& t, at::ScalarType type, int64_t n, void** o) {
  *o = nullptr;
  if (!t.defined()) return nullptr;
  if (!is_here(t)) return "an array lives on the current GPU";
  if (t.scalar_type() != type) return "an array has the wrong element type";
  if (t.numel() != n) return "an array has the wrong number of elements";
  if (!t.is_contiguous()) return "an array is contiguous";
  *o = t.data_ptr();
  return nullptr;
}
// What a caller handed over for it: None is an undefined tensor.
bool maybe_tensor(PyObject* o, Tensor& t) {
  if (o == Py_None) return true;
  if (!is_tensor(o)) return false;
  t = THPVariable_Unpack(o);
  return true;
}
// The arguments' tensors, from a[i0] on.
template <size_t N>
bool tensors_of(PyObject* const* a, Tensor (&t)[N]) {
  for (size_t i = 0; i < N; ++i)
    if (!maybe_tensor(a[i], t[i])) return false;
  return true;
}
#define ISP_REFUSE(what)                        \
  if (const char* bad_ = (what)) return fail(bad_)
#define ISP_REFUSE_IF(cond, what) \
  if (cond) return fail(what)

template <class F>
PyObject* call_free(Where w, F&& f) {  // a library call without a handle
  isp_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f(w.s);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}
// (workspaces: bytes on the current device)
const char* bytes_of(const Tensor& t, void** p, size_t* n) {
  *p = nullptr;
  *n = 0;
  if (!t.defined()) return nullptr;
  if (!is_here(t) || t.scalar_type() != at::kByte || !t.is_contiguous()) return "a workspace is a contiguous uint8 tensor on the current GPU";
  *p = t.data_ptr();
  *n = t.numel();
  return nullptr;
}

struct Norm {  // of the parameters
  void *w = nullptr, *b = nullptr;
  int type = ISP_F32;
};
const char* params_of(const Tensor& w, const Tensor& b, const Mat& X, Norm& o) {
  const Tensor& any = w.defined() ? w : b;
  if (!any.defined()) return nullptr;
  o.type = type_of(any.scalar_type());
  if (o.type != ISP_F32 && o.type != X.type) return "weight and bias are float32 or of the matrix's type";
  if (const char* bad = array_of(w, any.scalar_type(), X.d, &o.w)) return bad;
  return array_of(b, any.scalar_type(), X.d, &o.b);
}

// (X, Y, weight, bias, mean, rstd, eps, stream)
PyObject* py_layer_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(8)
  Tensor t[6];
  if (!is_tensor(a[0]) || !is_tensor(a[1]) || !tensors_of(a, t)) return nullptr;
  Mat X, Y;
  Norm P;
  void *mean, *rstd;
  ISP_REFUSE(mat_of(t[0], X));
  ISP_REFUSE(mat_of(t[1], Y));
  ISP_REFUSE_IF(Y.rows != X.rows || Y.d != X.d || Y.type != X.type, "X and Y have one shape and type");
  ISP_REFUSE(params_of(t[2], t[3], X, P));
  ISP_REFUSE(array_of(t[4], at::kFloat, X.rows, &mean));
  ISP_REFUSE(array_of(t[5], at::kFloat, X.rows, &rstd));
  const double eps = PyFloat_AsDouble(a[6]);
  const Where w = stream_of(a[7]);
  if (PyErr_Occurred()) return nullptr;
  return call_free(w, [&](void* s) {
    return isp_layer_norm(X.p, X.ld, X.rows, (int32_t)X.d, X.type, P.w, P.b, P.type, (float)eps, Y.p, Y.ld, (float*)mean, (float*)rstd, s);
  });
}

// (X, dY, dX, mean, rstd, weight, dweight, dbias, workspace, stream)
PyObject* py_layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(10)
  Tensor t[9];
  if (!is_tensor(a[0]) || !is_tensor(a[1]) || !tensors_of(a, t)) return nullptr;
  Mat X, G, O{nullptr, 0, 0, 0, 0};
  Norm P, D;
  void *mean, *rstd, *ws;
  size_t bytes;
  ISP_REFUSE(mat_of(t[0], X));
  ISP_REFUSE(mat_of(t[1], G));
  if (t[2].defined()) ISP_REFUSE(mat_of(t[2], O));
  ISP_REFUSE_IF(G.rows != X.rows || G.d != X.d || G.type != X.type, "X and dY have one shape and type");
  ISP_REFUSE_IF(t[2].defined() && (O.rows != X.rows || O.d != X.d || O.type != X.type), "X and dX have one shape and type");
  ISP_REFUSE_IF(!t[3].defined() || !t[4].defined(), "the backward needs the forward's mean and rstd");
  ISP_REFUSE(array_of(t[3], at::kFloat, X.rows, &mean));
  ISP_REFUSE(array_of(t[4], at::kFloat, X.rows, &rstd));
  ISP_REFUSE(params_of(t[5], Tensor(), X, P));
  ISP_REFUSE(params_of(t[6], t[7], X, D));
  ISP_REFUSE_IF(P.w && (D.w || D.b) && P.type != D.type, "the gradients of the parameters have the parameters' type");
  ISP_REFUSE(bytes_of(t[8], &ws, &bytes));
  const Where w = stream_of(a[9]);
  if (PyErr_Occurred()) return nullptr;
  return call_free(w, [&](void* s) {
    return isp_layer_norm_backward(X.p, X.ld, G.p, G.ld, X.rows, (int32_t)X.d, X.type, P.w, P.w ? P.type : D.type, (const float*)mean, (const float*)rstd,
                                   O.p, O.ld, D.w, D.b, ws, bytes, s);
  });
}

// (Z, labels, logprob, entropy, stats, top_logprob, top_index, workspace, stream)
PyObject* py_label_logprob(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(9)
  Tensor t[8];
  if (!is_tensor(a[0]) || !tensors_of(a, t)) return nullptr;
  Mat Z;
  void *labels, *lp, *en, *stats, *tv, *ti, *ws;
  size_t bytes;
  ISP_REFUSE(mat_of(t[0], Z));
  const Tensor& some = t[5].defined() ? t[5] : t[6];
  ISP_REFUSE_IF(some.defined() && (some.dim() != 2 || some.size(1) > Z.d), "the alternatives have one row per row of scores, of no more than its classes");
  const int64_t top = some.defined() ? some.size(1) : 0;
  ISP_REFUSE(array_of(t[1], at::kLong, Z.rows, &labels));
  ISP_REFUSE(array_of(t[2], at::kFloat, Z.rows, &lp));
  ISP_REFUSE(array_of(t[3], at::kFloat, Z.rows, &en));
  ISP_REFUSE(array_of(t[4], at::kFloat, 2 * Z.rows, &stats));
  ISP_REFUSE(array_of(t[5], at::kFloat, Z.rows * top, &tv));
  ISP_REFUSE(array_of(t[6], at::kInt, Z.rows * top, &ti));
  ISP_REFUSE(bytes_of(t[7], &ws, &bytes));
  const Where w = stream_of(a[8]);
  if (PyErr_Occurred()) return nullptr;
  return call_free(w, [&](void* s) {
    return isp_label_logprob(Z.p, Z.ld, Z.rows, (int32_t)Z.d, Z.type, (const int64_t*)labels, (float*)lp, (float*)en, (float*)stats, (int32_t)top, (float*)tv,
                             (int32_t*)ti, ws, bytes, s);
  });
}

// (Z, labels, stats, entropy, d_logprob, d_entropy, dZ, stream)
PyObject* py_label_logprob_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(8)
  Tensor t[7];
  if (!is_tensor(a[0]) || !is_tensor(a[6]) || !tensors_of(a, t)) return nullptr;
  Mat Z, O;
  void *labels, *stats, *en, *da, *de;
  ISP_REFUSE(mat_of(t[0], Z));
  ISP_REFUSE(mat_of(t[6], O));
  ISP_REFUSE_IF(O.rows != Z.rows || O.d != Z.d || O.type != Z.type, "Z and dZ have one shape and type");
  ISP_REFUSE(array_of(t[1], at::kLong, Z.rows, &labels));
  ISP_REFUSE(array_of(t[2], at::kFloat, 2 * Z.rows, &stats));
  ISP_REFUSE(array_of(t[3], at::kFloat, Z.rows, &en));
  ISP_REFUSE(array_of(t[4], at::kFloat, Z.rows, &da));
  ISP_REFUSE(array_of(t[5], at::kFloat, Z.rows, &de));
  const Where w = stream_of(a[7]);
  if (PyErr_Occurred()) return nullptr;
  return call_free(w, [&](void* s) {
    return isp_label_logprob_backward(Z.p, Z.ld, Z.rows, (int32_t)Z.d, Z.type, (const int64_t*)labels, (const float*)stats, (const float*)en, (const float*)da,
                                      (const float*)de, O.p, O.ld, s);
  });
}

struct Heads {
  int32_t heads, kv, dim;
};
const char* heads_of(const Cell& c, const Mat& Q, const Mat& K, const Mat& V, long heads, long kv, Heads& o) {
  if (heads <= 0 || kv <= 0 || heads > INT32_MAX || kv > INT32_MAX || Q.d % heads || Q.d == 0) return "Q's rows are `heads` heads of equal width";
  o.heads = (int32_t)heads;
  o.kv = (int32_t)kv;
  o.dim = (int32_t)(Q.d / heads);
  if (K.d != kv * o.dim || V.d != K.d) return "the rows of K and V are `kv_heads` heads of the width of Q's";
  if (Q.rows != c.n_rows || K.rows != c.n_cols || V.rows != K.rows) return "Q has A's rows, K and V its columns as rows";
  if (K.type != Q.type || V.type != Q.type) return "Q, K and V have one type";
  return nullptr;
}
bool same_shape(const Mat& a, const Mat& b) { return a.rows == b.rows && a.d == b.d && a.type == b.type; }

// (cell, Q, K, V, Y, stats, workspace, heads, kv_heads, scale, flags, stream)
PyObject* py_attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(12)
  Cell* c = cell_of(a[0]);
  Tensor t[6];
  for (int i = 1; i < 5; ++i)
    if (!c || !is_tensor(a[i])) return nullptr;
  if (!tensors_of(a + 1, t)) return nullptr;
  const long heads = PyLong_AsLong(a[7]), kv = PyLong_AsLong(a[8]);
  const double scale = PyFloat_AsDouble(a[9]);
  const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[10]);
  const Where w = stream_of(a[11]);
  if (PyErr_Occurred()) return nullptr;
  Mat Q, K, V, Y;
  Heads H;
  void *stats, *ws;
  size_t bytes;
  ISP_REFUSE(mat_of(t[0], Q));
  ISP_REFUSE(mat_of(t[1], K));
  ISP_REFUSE(mat_of(t[2], V));
  ISP_REFUSE(mat_of(t[3], Y));
  ISP_REFUSE(heads_of(*c, Q, K, V, heads, kv, H));
  ISP_REFUSE_IF(!same_shape(Q, Y), "Q and Y have one shape and type");
  ISP_REFUSE(array_of(t[4], at::kFloat, 2 * Q.rows * heads, &stats));
  ISP_REFUSE(bytes_of(t[5], &ws, &bytes));
  return call(c, w, [&](isp_csr_t* h, void* s) {
    return isp_attention(h, Q.p, Q.ld, K.p, K.ld, V.p, V.ld, H.heads, H.kv, H.dim, (float)scale, flags, Q.type, Y.p, Y.ld, (float*)stats, ws, bytes, s);
  });
}

// (cell, Q, K, V, stats, dY, dQ, dK, dV, workspace, heads, kv_heads, scale, flags, stream)
PyObject* py_attention_backward(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(15)
  Cell* c = cell_of(a[0]);
  Tensor t[9];
  for (int i = 1; i < 6; ++i)
    if (!c || !is_tensor(a[i])) return nullptr;
  if (!tensors_of(a + 1, t)) return nullptr;
  const long heads = PyLong_AsLong(a[10]), kv = PyLong_AsLong(a[11]);
  const double scale = PyFloat_AsDouble(a[12]);
  const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[13]);
  const Where w = stream_of(a[14]);
  if (PyErr_Occurred()) return nullptr;
  Mat Q, K, V, G, O[3] = {};
  Heads H;
  void *stats, *ws;
  size_t bytes;
  ISP_REFUSE(mat_of(t[0], Q));
  ISP_REFUSE(mat_of(t[1], K));
  ISP_REFUSE(mat_of(t[2], V));
  ISP_REFUSE(mat_of(t[4], G));
  ISP_REFUSE(heads_of(*c, Q, K, V, heads, kv, H));
  ISP_REFUSE_IF(!same_shape(Q, G), "Q and dY have one shape and type");
  for (int i = 0; i < 3; ++i)
    if (t[5 + i].defined()) {
      ISP_REFUSE(mat_of(t[5 + i], O[i]));
      ISP_REFUSE_IF(!same_shape(O[i], i == 0 ? Q : K), "a gradient has its operand's shape and type");
    }
  ISP_REFUSE(array_of(t[3], at::kFloat, 2 * Q.rows * heads, &stats));
  ISP_REFUSE(bytes_of(t[8], &ws, &bytes));
  return call(c, w, [&](isp_csr_t* h, void* s) {
    return isp_attention_backward(h, Q.p, Q.ld, K.p, K.ld, V.p, V.ld, H.heads, H.kv, H.dim, (float)scale, flags, Q.type, (const float*)stats, G.p, G.ld,
                                  O[0].p, O[0].ld, O[1].p, O[1].ld, O[2].p, O[2].ld, ws, bytes, s);
  });
}

// ---- autograd -------------------------------------------------------------------------------------------------
// The same operations as nodes of torch's graph.  The backward touches the interpreter only when a transpose has to
// be built or a call fails.  (4,096 rows, 32 columns, forward + backward: 112 -> 44 us of host time; a multiplication by
// a scalar takes 43 us in the same process: the rest is the engine's hand-over to its thread.)

// Raises binding.IspError for a status other than ISP_OK.
void check(isp_status st) {
  if (st == ISP_OK) return;
  pybind11::gil_scoped_acquire gil;
  PyObject* r = PyObject_CallFunction(g_check, "i", (int)st);
  Py_XDECREF(r);
  python_error e;
  e.persist();
  throw python_error(std::move(e));
}
// AssertionError, as the wrappers' own checks raise.
[[noreturn]] void assertion(const char* what) {
  pybind11::gil_scoped_acquire gil;
  PyErr_SetString(PyExc_AssertionError, what);
  python_error e;
  e.persist();
  throw python_error(std::move(e));
}
Dense dense(const Tensor& t) {
  Dense o;
  if (const char* bad = dense_of(t, o)) assertion(bad);
  return o;
}
// A library call on a cell's handle and the current stream.
template <class F>
void run(Cell& c, F&& f) {
  const Where w = here();
  const isp_status st = f(c.h.load(), w.s);
  if (st == ISP_OK || st == ISP_EHIP) c.ran_on(w);
  check(st);
}

// Everything the handle keeps of the values follows an in-place change of the tensor.
void sync_values(Graph& g) {
  if (!g.values.defined()) return;
  const uint32_t v = g.values._version();
  if (v == g.version) return;
  run(*g.A, [](isp_csr_t* h, void* s) { return isp_csr_values_changed(h, s); });
  g.version = v;
}

Cell& transpose(Graph& g) {
  sync_values(g);
  if (!g.At || !g.At->h.load()) {
    pybind11::gil_scoped_acquire gil;
    PyObject* r = PyObject_CallFunctionObjArgs(g_transpose, g.csr, nullptr);  // (At, was_cached)
    PyObject* cell = r ? PyObject_GetAttrString(PyTuple_GET_ITEM(r, 0), "_cell") : nullptr;
    if (cell) {
      if (auto* p = static_cast<CellPtr*>(PyCapsule_GetPointer(cell, CELL))) g.At = *p;
      Py_DECREF(cell);
    }
    Py_XDECREF(r);
    if (PyErr_Occurred()) {
      python_error e;
      e.persist();
      throw python_error(std::move(e));
    }
  }
  return *g.At;
}

Tensor new_like(const Tensor& t, int64_t rows, int64_t d) { return at::empty({rows, d}, t.options().requires_grad(false)); }

// No gradient here has a derivative of its own.  Asked for gradients that can be differentiated again (create_graph), a node hands them out with
// this one behind them, which says so to whoever goes through: otherwise their part of a second derivative would be lost without a word.
struct NoSecondDerivative : torch::autograd::Node {
  std::string name() const override { return "IspNoSecondDerivative"; }
  variable_list apply(variable_list&&) override {
    pybind11::gil_scoped_acquire gil;
    PyErr_SetString(PyExc_NotImplementedError, "the gradients of the sparse operations, layer norm, attention and label log probabilities cannot be differentiated again");
    python_error e;
    e.persist();
    throw python_error(std::move(e));
  }
};
// In a node's apply, made before anything else: the mode in which the engine runs it, and a mode without recording.
class Once {
  const bool again_ = at::GradMode::is_enabled();
  at::NoGradGuard no_grad_;

 public:
  // The gradients `out` of `grads`; by_input: they depend on the node's inputs, too.
  variable_list operator()(torch::autograd::Node& node, const variable_list& grads, variable_list out, bool by_input) const {
    if (!again_) return out;
    torch::autograd::edge_list edges = by_input ? node.next_edges() : torch::autograd::edge_list();
    for (const Tensor& g : grads)
      if (g.defined() && g.requires_grad()) edges.push_back(torch::autograd::impl::gradient_edge(g));
    if (std::none_of(edges.begin(), edges.end(), [](const torch::autograd::Edge& e) { return e.is_valid(); })) return out;
    auto stop = std::shared_ptr<NoSecondDerivative>(new NoSecondDerivative(), torch::autograd::deleteNode);
    stop->set_next_edges(std::move(edges));
    torch::autograd::set_history(out, stop);
    return out;
  }
};

struct SpmmBackward : torch::autograd::Node {
  GraphPtr graph;
  torch::autograd::SavedVariable X;  // only where the values have a gradient
  bool need_dA = false;
  std::string name() const override { return "IspSpmmBackward"; }
  void release_variables() override { X.reset_data(); }
  variable_list apply(variable_list&& grads) override {
    variable_list out(2);
    if (!grads[0].defined()) return out;
    const Once once;
    const Tensor dY = grads[0].contiguous();
    const Dense G = dense(dY);
    if (task_should_compute_output(1)) {
      out[1] = new_like(dY, graph->A->n_cols, G.d);
      const Dense O = dense(out[1]);
      run(transpose(*graph), [&](isp_csr_t* h, void* s) { return isp_spmm(h, G.p, G.ld, (int32_t)G.d, O.p, O.ld, s); });
    }
    if (need_dA && task_should_compute_output(0)) {
      const Tensor x = X.unpack();
      const Dense V = dense(x);
      out[0] = at::empty({graph->A->nnz}, dY.options());
      run(*graph->A, [&](isp_csr_t* h, void* s) { return isp_sddmm(h, G.p, G.ld, V.p, V.ld, (int32_t)G.d, 0, static_cast<float*>(out[0].data_ptr()), s); });
    }
    return once(*this, grads, std::move(out), need_dA);
  }
};

struct ReduceBackward : torch::autograd::Node {
  GraphPtr graph;
  int reduce = 0;
  Tensor arg;
  std::string name() const override { return "IspSpmmReduceBackward"; }
  variable_list apply(variable_list&& grads) override {
    variable_list out(1);
    if (!grads[0].defined()) return out;
    const Once once;
    transpose(*graph);  // built on the first backward, cached afterwards
    const Tensor dY = grads[0].contiguous();
    const Dense G = dense(dY);
    out[0] = new_like(dY, graph->A->n_cols, G.d);
    const Dense O = dense(out[0]);
    run(*graph->A, [&](isp_csr_t* h, void* s) {
      return isp_spmm_reduce_backward(h, G.p, G.ld, (int32_t)G.d, reduce, arg.defined() ? static_cast<const int32_t*>(arg.data_ptr()) : nullptr, O.p, O.ld, s);
    });
    return once(*this, grads, std::move(out), false);
  }
};

struct FusedBackward : torch::autograd::Node {
  GraphPtr graph;
  torch::autograd::SavedVariable X;
  std::string name() const override { return "IspFusedmmBackward"; }
  void release_variables() override { X.reset_data(); }
  variable_list apply(variable_list&& grads) override {
    variable_list out(1);
    if (!grads[0].defined()) return out;
    const Once once;
    transpose(*graph);
    const Tensor x = X.unpack(), dY = grads[0].contiguous();
    const Dense V = dense(x), G = dense(dY);
    out[0] = new_like(x, V.rows, V.d);
    const Dense O = dense(out[0]);
    run(*graph->A, [&](isp_csr_t* h, void* s) { return isp_fusedmm_backward(h, V.p, V.ld, G.p, G.ld, (int32_t)V.d, ISP_OP_SIGMOID, O.p, O.ld, s); });
    return once(*this, grads, std::move(out), true);
  }
};

// The nodes have no forward-mode rule: a tangent would be lost without a word.
bool no_tangent(const Tensor& t) {
  if (!t.defined() || !t._fw_grad(/*level=*/0).defined()) return true;
  PyErr_SetString(PyExc_NotImplementedError, "the sparse operations have no forward-mode derivative");
  return false;
}

GraphPtr graph_of(PyObject* c) {
  auto* p = static_cast<GraphPtr*>(PyCapsule_GetPointer(c, GRAPH));
  if (!p) throw python_error();
  return *p;
}

// (cell of A, the CSR object, values or None) -> graph
PyObject* py_graph(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(3)
  auto* c = static_cast<CellPtr*>(PyCapsule_GetPointer(a[0], CELL));
  if (!c || (a[2] != Py_None && !is_tensor(a[2]))) return nullptr;
  auto g = std::make_shared<Graph>();
  g->A = *c;
  Py_INCREF(a[1]);
  g->csr = a[1];
  if (a[2] != Py_None) {
    g->values = THPVariable_Unpack(a[2]);
    g->version = g->values._version();
  }
  return wrap(std::move(g), GRAPH);
  END_HANDLE_TH_ERRORS
}

PyObject* py_graph_sync(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(1)
  sync_values(*graph_of(a[0]));
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// (graph, values or None, X) -> Y = A X
PyObject* py_ag_spmm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(3)
  GraphPtr g = graph_of(a[0]);
  if ((a[1] != Py_None && !is_tensor(a[1])) || !is_tensor(a[2])) return nullptr;
  const Tensor values = a[1] == Py_None ? Tensor() : THPVariable_Unpack(a[1]);
  const Tensor x = THPVariable_Unpack(a[2]);
  if (!no_tangent(values) || !no_tangent(x)) return nullptr;
  Tensor Y;
  {
    pybind11::gil_scoped_release release;
    Tensor xc;
    {
      at::NoGradGuard no_grad;
      xc = x.contiguous();
      const Dense X = dense(xc);
      if (X.rows != g->A->n_cols) assertion("X has A's columns as rows");
      Y = new_like(xc, g->A->n_rows, X.d);
      const Dense O = dense(Y);
      sync_values(*g);
      run(*g->A, [&](isp_csr_t* h, void* s) { return isp_spmm(h, X.p, X.ld, (int32_t)X.d, O.p, O.ld, s); });
    }
    if (torch::autograd::compute_requires_grad(values, x)) {
      auto node = std::shared_ptr<SpmmBackward>(new SpmmBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(values, x));
      node->graph = g;
      node->need_dA = values.defined() && values.requires_grad();
      if (node->need_dA) node->X = torch::autograd::SavedVariable(xc, false);
      torch::autograd::set_history(Y, node);
    }
  }
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// (graph, X, reduce) -> Y of mean / min / max
PyObject* py_ag_reduce(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(3)
  GraphPtr g = graph_of(a[0]);
  if (!is_tensor(a[1])) return nullptr;
  const Tensor x = THPVariable_Unpack(a[1]);
  if (!no_tangent(x)) return nullptr;
  const int reduce = (int)PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  Tensor Y, arg;
  {
    pybind11::gil_scoped_release release;
    {
      at::NoGradGuard no_grad;
      const Tensor xc = x.contiguous();
      const Dense X = dense(xc);
      if (X.rows != g->A->n_cols) assertion("X has A's columns as rows");
      Y = new_like(xc, g->A->n_rows, X.d);
      if (reduce != ISP_REDUCE_MEAN) arg = at::empty({g->A->n_rows, X.d}, Y.options().dtype(at::kInt));
      const Dense O = dense(Y);
      sync_values(*g);
      run(*g->A, [&](isp_csr_t* h, void* s) {
        return isp_spmm_reduce(h, X.p, X.ld, (int32_t)X.d, reduce, O.p, O.ld, arg.defined() ? static_cast<int32_t*>(arg.data_ptr()) : nullptr, s);
      });
    }
    if (torch::autograd::compute_requires_grad(x)) {
      auto node = std::shared_ptr<ReduceBackward>(new ReduceBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(x));
      node->graph = g;
      node->reduce = reduce;
      node->arg = arg;
      torch::autograd::set_history(Y, node);
    }
  }
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// (graph, X) -> Y of the sigmoid FusedMM
PyObject* py_ag_fused(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(2)
  GraphPtr g = graph_of(a[0]);
  if (!is_tensor(a[1])) return nullptr;
  const Tensor x = THPVariable_Unpack(a[1]);
  if (!no_tangent(x)) return nullptr;
  Tensor Y;
  {
    pybind11::gil_scoped_release release;
    Tensor xc;
    {
      at::NoGradGuard no_grad;
      xc = x.contiguous();
      const Dense X = dense(xc);
      if (X.rows != g->A->n_rows) assertion("X has A's rows");
      Y = new_like(xc, X.rows, X.d);
      const Dense O = dense(Y);
      sync_values(*g);
      run(*g->A, [&](isp_csr_t* h, void* s) { return isp_fusedmm(h, X.p, X.ld, (int32_t)X.d, ISP_OP_SIGMOID, O.p, O.ld, s); });
    }
    if (torch::autograd::compute_requires_grad(x)) {
      auto node = std::shared_ptr<FusedBackward>(new FusedBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(x));
      node->graph = g;
      node->X = torch::autograd::SavedVariable(xc, false);
      torch::autograd::set_history(Y, node);
    }
  }
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// ---- the row-wise operators' nodes -------------------------------------------------------------------------------------
Mat mat(const Tensor& t) {
  Mat o;
  if (const char* bad = mat_of(t, o)) assertion(bad);
  return o;
}
void* array(const Tensor& t, at::ScalarType type, int64_t n) {
  void* p;
  if (const char* bad = array_of(t, type, n, &p)) assertion(bad);
  return p;
}
Norm params(const Tensor& w, const Tensor& b, const Mat& X) {
  Norm o;
  if (const char* bad = params_of(w, b, X, o)) assertion(bad);
  return o;
}
Tensor rows_of(const Tensor& t) { return t.dim() == 2 && t.stride(1) == 1 && (t.size(0) < 2 || t.stride(0) >= t.size(1)) ? t : t.contiguous(); }
Tensor floats_like(const Tensor& t, at::IntArrayRef shape) { return at::empty(shape, t.options().dtype(at::kFloat).requires_grad(false)); }
Tensor workspace_like(const Tensor& t, size_t bytes) { return at::empty({(int64_t)bytes}, t.options().dtype(at::kByte).requires_grad(false)); }
using torch::autograd::SavedVariable;

struct LayerNormBackward : torch::autograd::Node {
  SavedVariable X, weight;
  Tensor mean, rstd;
  bool bias = false;
  std::vector<int64_t> bias_shape;  // (any shape of d elements)
  at::ScalarType param = at::kFloat;
  std::string name() const override { return "IspLayerNormBackward"; }
  void release_variables() override {
    X.reset_data();
    weight.reset_data();
    mean.reset();
    rstd.reset();
  }
  variable_list apply(variable_list&& grads) override {
    variable_list out(3);
    if (!grads[0].defined()) return out;
    const Once once;
    const Tensor x = X.unpack(), w = weight.unpack(), dY = rows_of(grads[0]);
    const Mat M = mat(x), G = mat(dY);
    const Norm P = params(w, Tensor(), M);
    Mat O{nullptr, 0, 0, 0, 0};
    if (task_should_compute_output(0)) {
      out[0] = at::empty({M.rows, M.d}, x.options().requires_grad(false));
      O = mat(out[0]);
    }
    const auto like = x.options().dtype(param).requires_grad(false);
    if (P.w && task_should_compute_output(1)) out[1] = at::empty(w.sizes(), like);
    if (bias && task_should_compute_output(2)) out[2] = at::empty(bias_shape, like);
    size_t bytes = 0;
    Tensor ws;
    if (out[1].defined() || out[2].defined()) {
      check(isp_layer_norm_backward_workspace(M.rows, (int32_t)M.d, &bytes));
      ws = workspace_like(x, bytes);
    }
    check(isp_layer_norm_backward(M.p, M.ld, G.p, G.ld, M.rows, (int32_t)M.d, M.type, P.w, type_of(param), mean.data_ptr<float>(), rstd.data_ptr<float>(),
                                  O.p, O.ld, out[1].defined() ? out[1].data_ptr() : nullptr, out[2].defined() ? out[2].data_ptr() : nullptr,
                                  ws.defined() ? ws.data_ptr() : nullptr, bytes, here().s));
    return once(*this, grads, std::move(out), true);
  }
};

// (X, weight or None, bias or None, eps) -> Y
PyObject* py_ag_layer_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(4)
  Tensor t[3];
  if (!is_tensor(a[0]) || !tensors_of(a, t)) return nullptr;
  const double eps = PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) return nullptr;
  for (const Tensor& v : t)
    if (!no_tangent(v)) return nullptr;
  Tensor Y;
  {
    pybind11::gil_scoped_release release;
    Tensor x, w, b, mean, rstd;
    const bool grad = torch::autograd::compute_requires_grad(t[0], t[1], t[2]);
    Norm P;
    {
      at::NoGradGuard no_grad;
      x = rows_of(t[0]);
      if (t[1].defined()) w = t[1].contiguous();
      if (t[2].defined()) b = t[2].contiguous();
      const Mat X = mat(x);
      P = params(w, b, X);
      Y = at::empty({X.rows, X.d}, x.options().requires_grad(false));
      const Mat O = mat(Y);
      if (grad) {
        mean = floats_like(x, {X.rows});
        rstd = floats_like(x, {X.rows});
      }
      check(isp_layer_norm(X.p, X.ld, X.rows, (int32_t)X.d, X.type, P.w, P.b, P.type, (float)eps, O.p, O.ld, grad ? mean.data_ptr<float>() : nullptr,
                           grad ? rstd.data_ptr<float>() : nullptr, here().s));
    }
    if (grad) {
      auto node = std::shared_ptr<LayerNormBackward>(new LayerNormBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(t[0], t[1], t[2]));
      node->X = SavedVariable(x, false);
      if (w.defined()) node->weight = SavedVariable(w, false);
      node->mean = mean;
      node->rstd = rstd;
      node->bias = b.defined();
      if (b.defined()) node->bias_shape = b.sizes().vec();
      node->param = P.type == ISP_F32 ? at::kFloat : x.scalar_type();
      torch::autograd::set_history(Y, node);
    }
  }
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

struct LabelLogprobBackward : torch::autograd::Node {
  SavedVariable Z, labels, entropy;
  Tensor stats;
  std::string name() const override { return "IspLabelLogprobBackward"; }
  void release_variables() override {
    Z.reset_data();
    labels.reset_data();
    entropy.reset_data();
    stats.reset();
  }
  variable_list apply(variable_list&& grads) override {
    variable_list out(1);
    if (!grads[0].defined() && !grads[1].defined()) return out;
    const Once once;
    const Tensor z = Z.unpack(), y = labels.unpack(), e = entropy.unpack(shared_from_this());
    const Mat M = mat(z);
    const Tensor da = grads[0].defined() ? grads[0].contiguous() : Tensor(), de = grads[1].defined() ? grads[1].contiguous() : Tensor();
    out[0] = at::empty({M.rows, M.d}, z.options().requires_grad(false));
    const Mat O = mat(out[0]);
    check(isp_label_logprob_backward(M.p, M.ld, M.rows, (int32_t)M.d, M.type, static_cast<const int64_t*>(array(y, at::kLong, M.rows)), stats.data_ptr<float>(),
                                     static_cast<const float*>(array(e, at::kFloat, M.rows)), static_cast<const float*>(array(da, at::kFloat, M.rows)),
                                     static_cast<const float*>(array(de, at::kFloat, M.rows)), O.p, O.ld, here().s));
    return once(*this, grads, std::move(out), true);
  }
};

// (Z, labels, top) -> (logprob, entropy) or, with top > 0, (logprob, entropy, top_logprob, top_index)
PyObject* py_ag_label_logprob(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(3)
  if (!is_tensor(a[0]) || !is_tensor(a[1])) return nullptr;
  const Tensor Z = THPVariable_Unpack(a[0]), labels = THPVariable_Unpack(a[1]);
  const long top = PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  if (!no_tangent(Z)) return nullptr;
  Tensor lp, en, tv, ti;
  {
    pybind11::gil_scoped_release release;
    const bool grad = torch::autograd::compute_requires_grad(Z);
    Tensor z, y, stats;
    {
      at::NoGradGuard no_grad;
      z = rows_of(Z);
      y = labels.contiguous();
      const Mat M = mat(z);
      if (top < 0 || top > M.d) assertion("top is not in [0, classes]");
      const auto* L = static_cast<const int64_t*>(array(y, at::kLong, M.rows));
      lp = floats_like(z, {M.rows});
      en = floats_like(z, {M.rows});
      if (grad) stats = floats_like(z, {M.rows, 2});
      if (top > 0) {
        tv = floats_like(z, {M.rows, top});
        ti = at::empty({M.rows, top}, tv.options().dtype(at::kInt));
      }
      size_t bytes = 0;
      check(isp_label_logprob_workspace(M.rows, (int32_t)M.d, (int32_t)top, &bytes));
      Tensor ws;
      if (bytes) ws = workspace_like(z, bytes);
      check(isp_label_logprob(M.p, M.ld, M.rows, (int32_t)M.d, M.type, L, lp.data_ptr<float>(), en.data_ptr<float>(), grad ? stats.data_ptr<float>() : nullptr,
                              (int32_t)top, top > 0 ? tv.data_ptr<float>() : nullptr, top > 0 ? ti.data_ptr<int32_t>() : nullptr,
                              bytes ? ws.data_ptr() : nullptr, bytes, here().s));
    }
    if (grad) {
      auto node = std::shared_ptr<LabelLogprobBackward>(new LabelLogprobBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(Z));
      node->Z = SavedVariable(z, false);
      node->labels = SavedVariable(y, false);
      node->stats = stats;
      torch::autograd::set_history(lp, node);
      torch::autograd::set_history(en, node);
      node->entropy = SavedVariable(en, true);
    }
  }
  return top > 0 ? Py_BuildValue("(NNNN)", THPVariable_Wrap(lp), THPVariable_Wrap(en), THPVariable_Wrap(tv), THPVariable_Wrap(ti))
                 : Py_BuildValue("(NN)", THPVariable_Wrap(lp), THPVariable_Wrap(en));
  END_HANDLE_TH_ERRORS
}

struct AttentionBackward : torch::autograd::Node {
  GraphPtr graph;
  SavedVariable Q, K, V;
  Tensor stats;
  Heads H{};
  float scale = 0.f;
  unsigned flags = 0;
  uint32_t bias_version = 0;  // of the graph's values, where they take part
  std::string name() const override { return "IspAttentionBackward"; }
  void release_variables() override {
    for (SavedVariable* v : {&Q, &K, &V}) v->reset_data();
    stats.reset();
  }
  variable_list apply(variable_list&& grads) override {
    variable_list out(3);
    if (!grads[0].defined()) return out;
    const Once once;
    TORCH_CHECK(!(flags & ISP_BIAS_BY_A) || graph->values._version() == bias_version,
                "the graph's values, which the attention's backward needs, have been modified by an inplace operation");
    const Tensor q = Q.unpack(), k = K.unpack(), v = V.unpack(), dY = rows_of(grads[0]);
    const bool rows = task_should_compute_output(0), cols = task_should_compute_output(1) || task_should_compute_output(2);
    if (cols) transpose(*graph);
    else sync_values(*graph);
    const Mat MQ = mat(q), MK = mat(k), MV = mat(v), G = mat(dY);
    Mat O[3] = {};
    if (rows) {
      out[0] = at::empty({MQ.rows, MQ.d}, q.options().requires_grad(false));
      O[0] = mat(out[0]);
    }
    if (cols)
      for (int i = 1; i < 3; ++i) {
        out[i] = at::empty({MK.rows, MK.d}, k.options().requires_grad(false));
        O[i] = mat(out[i]);
      }
    size_t bytes = 0;
    check(isp_attention_backward_workspace(graph->A->h.load(), H.heads, H.kv, H.dim, &bytes));
    const Tensor ws = workspace_like(q, bytes);
    run(*graph->A, [&](isp_csr_t* h, void* s) {
      return isp_attention_backward(h, MQ.p, MQ.ld, MK.p, MK.ld, MV.p, MV.ld, H.heads, H.kv, H.dim, scale, flags, MQ.type, stats.data_ptr<float>(),
                                    G.p, G.ld, O[0].p, O[0].ld, O[1].p, O[1].ld, O[2].p, O[2].ld, ws.data_ptr(), bytes, s);
    });
    return once(*this, grads, std::move(out), true);
  }
};

// (graph, Q, K, V, heads, kv_heads, scale or None, flags) -> Y
PyObject* py_ag_attention(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  ISP_ARGS(8)
  GraphPtr g = graph_of(a[0]);
  for (int i = 1; i < 4; ++i)
    if (!is_tensor(a[i])) return nullptr;
  Tensor t[3];
  if (!tensors_of(a + 1, t)) return nullptr;
  const long heads = PyLong_AsLong(a[4]), kv = PyLong_AsLong(a[5]);
  double scale = a[6] == Py_None ? 0. : PyFloat_AsDouble(a[6]);
  const unsigned flags = (unsigned)PyLong_AsUnsignedLong(a[7]);
  if (PyErr_Occurred()) return nullptr;
  for (const Tensor& v : t)
    if (!no_tangent(v)) return nullptr;
  Tensor Y;
  {
    pybind11::gil_scoped_release release;
    const bool grad = torch::autograd::compute_requires_grad(t[0], t[1], t[2]);
    Tensor q, k, v, stats;
    Heads H;
    {
      at::NoGradGuard no_grad;
      q = rows_of(t[0]);
      k = rows_of(t[1]);
      v = rows_of(t[2]);
      const Mat MQ = mat(q), MK = mat(k), MV = mat(v);
      if (const char* bad = heads_of(*g->A, MQ, MK, MV, heads, kv, H)) assertion(bad);
      if (a[6] == Py_None) scale = 1. / std::sqrt((double)H.dim);
      Y = at::empty({MQ.rows, MQ.d}, q.options().requires_grad(false));
      const Mat O = mat(Y);
      if (grad) stats = floats_like(q, {MQ.rows, heads, 2});
      size_t bytes = 0;
      check(isp_attention_workspace(g->A->h.load(), H.heads, H.kv, H.dim, MQ.type, &bytes));
      Tensor ws;
      if (bytes) ws = workspace_like(q, bytes);
      sync_values(*g);
      run(*g->A, [&](isp_csr_t* h, void* s) {
        return isp_attention(h, MQ.p, MQ.ld, MK.p, MK.ld, MV.p, MV.ld, H.heads, H.kv, H.dim, (float)scale, flags, MQ.type, O.p, O.ld,
                             grad ? stats.data_ptr<float>() : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, s);
      });
    }
    if (grad) {
      auto node = std::shared_ptr<AttentionBackward>(new AttentionBackward(), torch::autograd::deleteNode);
      node->set_next_edges(torch::autograd::collect_next_edges(t[0], t[1], t[2]));
      node->graph = g;
      node->Q = SavedVariable(q, false);
      node->K = SavedVariable(k, false);
      node->V = SavedVariable(v, false);
      node->stats = stats;
      node->H = H;
      node->scale = (float)scale;
      node->flags = flags;
      if (flags & ISP_BIAS_BY_A) node->bias_version = g->version;
      torch::autograd::set_history(Y, node);
    }
  }
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// (binding._check, binding.csr_transpose_cached)
PyObject* py_init(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  ISP_ARGS(2)
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  g_check = a[0];
  g_transpose = a[1];
  Py_RETURN_NONE;
}

// No C++ exception leaves an entry point: asking some tensors (vmap's, sparse ones) for strides or storage throws.
template <PyObject* (*FN)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  try {
    return FN(self, a, nargs);
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

#define ISP_DEF(name, fn) {name, (PyCFunction)(void (*)(void))(PyObject * (*)(PyObject*, PyObject* const*, Py_ssize_t)) guarded<fn>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ISP_DEF("init", py_init),
    ISP_DEF("cell", py_cell),
    ISP_DEF("cell_clear", py_cell_clear),
    ISP_DEF("cell_ran", py_cell_ran),
    ISP_DEF("cell_foreign", py_cell_foreign),
    ISP_DEF("cells_release", py_cells_release),
    ISP_DEF("spmm", py_spmm<isp_spmm>),
    ISP_DEF("spmm_static_scratch", py_spmm<isp_spmm_static_scratch>),
    ISP_DEF("sddmm", py_sddmm),
    ISP_DEF("fusedmm", py_fusedmm),
    ISP_DEF("fusedmm_backward", py_fusedmm_backward),
    ISP_DEF("spmm_reduce", py_spmm_reduce),
    ISP_DEF("spmm_reduce_backward", py_spmm_reduce_backward),
    ISP_DEF("layer_norm", py_layer_norm),
    ISP_DEF("layer_norm_backward", py_layer_norm_backward),
    ISP_DEF("label_logprob", py_label_logprob),
    ISP_DEF("label_logprob_backward", py_label_logprob_backward),
    ISP_DEF("ag_layer_norm", py_ag_layer_norm),
    ISP_DEF("ag_label_logprob", py_ag_label_logprob),
    ISP_DEF("attention", py_attention),
    ISP_DEF("attention_backward", py_attention_backward),
    ISP_DEF("ag_attention", py_ag_attention),
    ISP_DEF("graph", py_graph),
    ISP_DEF("graph_sync", py_graph_sync),
    ISP_DEF("ag_spmm", py_ag_spmm),
    ISP_DEF("ag_reduce", py_ag_reduce),
    ISP_DEF("ag_fused", py_ag_fused),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_isp_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__isp_torch() { return PyModule_Create(&module); }
