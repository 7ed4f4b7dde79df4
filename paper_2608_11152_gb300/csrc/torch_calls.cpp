// The KV operators' calls on torch tensors: checks of the arguments, the result's memory, the current
// stream, and the C entry point, in one step.
//
// These calls are made once a layer and token.  Through ctypes the same steps took 9 us of a call whose
// kernel takes 3 (torch.empty 3.3, checks and attribute reads 1.8, argument conversion 1.5, launch 2.1).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <vector>

#include "../../include/misat.h"

namespace {

PyObject* g_error = nullptr;  // MisatError

struct Rope {
  static constexpr const char* kName = "Rope";
  misat_rope* h;
  c10::DeviceIndex device;
};
struct Pool {
  static constexpr const char* kName = "KvPool";
  misat_kv* h;
  c10::DeviceIndex device;
  at::Tensor k_blocks, v_blocks;
  at::ScalarType dtype;
  int64_t hq, hkv, d;
  cudaStream_t last;  // of the last call outside a capture
  bool called;
};
// Tensors that a call made for later ones: these may run on another stream.
struct Made {
  cudaStream_t on;
  std::vector<at::Tensor> tensors;
};
struct Batch {
  static constexpr const char* kName = "KvBatch";
  misat_kv_batch b;
  int64_t hq, hkv, d;
  c10::DeviceIndex device;
  Made made{};
};
struct Tree {
  static constexpr const char* kName = "KvTree";
  misat_kv_draft d;
  int64_t n_tokens, max_q;
  c10::DeviceIndex device;
  Made made;
};
struct Norm {
  static constexpr const char* kName = "HeadNorm";
  at::Tensor w;  // [head_dim] or [heads][head_dim]
  float eps, offset;
};

template <class S>
void free_state(PyObject* c) {
  delete static_cast<S*>(PyCapsule_GetPointer(c, S::kName));
}
template <class S>
PyObject* new_state(const S& s) {
  S* p = new S(s);
  PyObject* c = PyCapsule_New(p, S::kName, free_state<S>);
  if (!c) delete p;
  return c;
}
// The state behind an object of the binding; nullptr with an error set for another kind's.
template <class S>
S* state(PyObject* c) {
  return static_cast<S*>(PyCapsule_GetPointer(c, S::kName));
}

struct Raised {};  // a Python error is set

PyObject* fail(int code, const char* where) {
  PyObject* e = PyObject_CallFunction(g_error, "is", code, where);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}

[[noreturn]] void refuse(const char* name, const std::string& expected, const at::Tensor& t) {
  std::ostringstream s;
  s << name << ": " << expected << " expected, got " << t.scalar_type() << " " << t.sizes() << " on " << t.device();
  PyErr_SetString(PyExc_ValueError, s.str().c_str());
  throw Raised{};
}
const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s: a tensor expected", name);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}
// A tensor [tokens][heads][head_dim] whose heads are contiguous.
const at::Tensor& heads(PyObject* o, const char* name, at::ScalarType dtype, c10::DeviceIndex device, int64_t n,
                        int64_t h, int64_t d) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != dtype || !t.is_cuda() || t.get_device() != device || t.dim() != 3 || t.size(0) != n ||
      t.size(1) != h || t.size(2) != d || (d > 1 && t.stride(2) != 1)) {
    std::ostringstream s;
    s << dtype << " [" << n << ", " << h << ", " << d << "] on cuda:" << (int)device << " with contiguous heads";
    refuse(name, s.str(), t);
  }
  return t;
}
at::Tensor fresh(at::IntArrayRef size, at::ScalarType dtype, c10::DeviceIndex device) {
  return at::Tensor(at::detail::empty_cuda(size, dtype, at::Device(at::kCUDA, device), std::nullopt));
}
// A tensor of whole numbers in an array of them, from number `from` (of the tensor's type) on: an allocation is 0.7 us,
// this 0.1.
at::Tensor piece(const at::Tensor& array, int64_t from, at::IntArrayRef size, at::ScalarType dtype = at::kInt) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(array.storage()), array.key_set(),
                                                          c10::scalarTypeToTypeMeta(dtype));
  t.unsafeGetTensorImpl()->set_storage_offset(from);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
  return t;
}
// Autograd finds out by its version that a tensor it has saved was written.
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// A contiguous tensor of whole numbers.
template <class I = int32_t>
I* ints(const at::Tensor& t, const char* name, c10::DeviceIndex device, std::initializer_list<int64_t> size) {
  constexpr bool kWide = sizeof(I) == 8;
  if (t.scalar_type() != (kWide ? at::kLong : at::kInt) || !t.is_cuda() || t.get_device() != device ||
      !t.sizes().equals(size) || !t.is_contiguous()) {
    std::ostringstream s;
    s << "contiguous " << (kWide ? "int64 " : "int32 ") << at::IntArrayRef(size) << " on cuda:" << (int)device;
    refuse(name, s.str(), t);
  }
  return t.data_ptr<I>();
}
// A block table [n][columns]: its columns.
int64_t table_columns(const at::Tensor& t, c10::DeviceIndex device, int64_t n, int64_t& stride) {
  const bool shaped = t.scalar_type() == at::kInt && t.is_cuda() && t.get_device() == device && t.dim() == 2 &&
                      t.size(0) == n;
  const int64_t columns = shaped ? t.size(1) : 0;
  stride = shaped && n > 1 ? t.stride(0) : columns;
  if (!shaped || (columns > 1 && t.stride(1) != 1) || stride < columns)
    refuse("block_table",
           "int32 [" + std::to_string(n) + ", blocks] on cuda:" + std::to_string((int)device) +
               " with contiguous rows that do not overlap",
           t);
  return columns;
}
int32_t int32_of(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < INT32_MIN || v > INT32_MAX) {
    PyErr_Format(PyExc_ValueError, "%s: beyond 32 bits", name);
    throw Raised{};
  }
  return (int32_t)v;
}

int code_of(at::ScalarType t) {
  return t == at::kBFloat16 ? MISAT_BF16 : t == at::kHalf ? MISAT_F16 : t == at::kFloat ? MISAT_F32 : -1;
}

bool capturing(cudaStream_t st) {
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusActive;
  return cudaStreamIsCapturing(st, &status) != cudaSuccess || status != cudaStreamCaptureStatusNone;
}
// The current stream; a pool's calls share its workspace, so a change of stream waits for the calls on
// the last one.  Under capture nothing is recorded: whoever replays the graph orders it with other calls.
// Where the last stream cannot be waited for (it is being captured, or gone), the call is an error.
cudaStream_t ordered(Pool* p) {
  const cudaStream_t st = c10::cuda::getCurrentCUDAStream(p->device).stream();
  if ((p->called && st == p->last) || capturing(st)) return st;
  if (p->called) {
    cudaEvent_t e = nullptr;
    bool ok = !capturing(p->last) && cudaEventCreateWithFlags(&e, cudaEventDisableTiming) == cudaSuccess;
    ok = ok && cudaEventRecord(e, p->last) == cudaSuccess && cudaStreamWaitEvent(st, e, 0) == cudaSuccess;
    if (e) cudaEventDestroy(e);
    if (!ok) {
      cudaGetLastError();
      fail(MISAT_ERR_STATE, "KvPool: the stream of its last call cannot be waited for");
      throw Raised{};
    }
  }
  p->called = true;
  p->last = st;
  return st;
}

#define MISAT_TRY HANDLE_TH_ERRORS try {
#define MISAT_END                 \
  }                               \
  catch (const Raised&) {         \
    return nullptr;               \
  }                               \
  END_HANDLE_TH_ERRORS

bool count(Py_ssize_t n, Py_ssize_t expected) {
  if (n != expected) PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", expected, n);
  return n == expected;
}

// (error class)
PyObject* init(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  g_error = cls;
  Py_RETURN_NONE;
}

// (handle, device)
PyObject* rope_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 2)) return nullptr;
  Rope r{static_cast<misat_rope*>(PyLong_AsVoidPtr(a[0])), (c10::DeviceIndex)PyLong_AsLong(a[1])};
  return PyErr_Occurred() ? nullptr : new_state(r);
  MISAT_END
}

// (handle, device, k_blocks, v_blocks, q heads)
PyObject* pool_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 5)) return nullptr;
  const at::Tensor &k = tensor(a[2], "k_blocks"), &v = tensor(a[3], "v_blocks");
  Pool p{static_cast<misat_kv*>(PyLong_AsVoidPtr(a[0])), (c10::DeviceIndex)PyLong_AsLong(a[1]), k, v, k.scalar_type(),
         PyLong_AsLong(a[4]), k.size(1), k.size(3), nullptr, false};
  return PyErr_Occurred() ? nullptr : new_state(p);
  MISAT_END
}

// (pool, q_off, kv_len, block_table, n_tokens, max_q)
PyObject* batch_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 6)) return nullptr;
  const Pool* p = state<Pool>(a[0]);
  if (!p) return nullptr;
  const at::Tensor &off = tensor(a[1], "q_off"), &len = tensor(a[2], "kv_len"), &table = tensor(a[3], "block_table");
  const int64_t seqs = len.dim() == 1 ? len.size(0) : 0;
  int64_t stride;
  ints(len, "kv_len", p->device, {seqs});
  ints(off, "q_off", p->device, {seqs + 1});
  table_columns(table, p->device, seqs, stride);
  const long long tokens = PyLong_AsLongLong(a[4]), max_q = PyLong_AsLongLong(a[5]);
  if (PyErr_Occurred()) return nullptr;
  if (seqs > INT32_MAX || tokens < INT32_MIN || tokens > INT32_MAX || max_q < INT32_MIN || max_q > INT32_MAX)
    return fail(MISAT_ERR_INVALID_ARG, "misat_kv_batch");
  Batch b{{(int32_t)seqs, (int32_t)tokens, (int32_t)max_q, off.data_ptr<int32_t>(), len.data_ptr<int32_t>(),
           table.data_ptr<int32_t>(), stride},
          p->hq, p->hkv, p->d, p->device};
  return new_state(b);
  MISAT_END
}

// A later call on the tensors that an earlier one made: their memory is not used again before it is finished.
void used(const Made& m, cudaStream_t st) {
  if (m.tensors.empty() || m.on == st || capturing(st)) return;
  for (const at::Tensor& t : m.tensors)
    c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), c10::cuda::getCurrentCUDAStream(t.get_device()));
}

// (rope, x, positions, out or None, backward) -> out
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 5)) return nullptr;
  const Rope* r = state<Rope>(a[0]);
  if (!r) return nullptr;
  const at::Tensor& x = tensor(a[1], "x");
  const int code = code_of(x.scalar_type());
  if (code < 0 || x.dim() != 3) refuse("x", "[tokens, heads, head_dim] of bfloat16, float16 or float32", x);
  const int64_t T = x.size(0), H = x.size(1), D = x.size(2);
  heads(a[1], "x", x.scalar_type(), r->device, T, H, D);
  const at::Tensor& pos = tensor(a[2], "positions");
  if (pos.scalar_type() != at::kInt || !pos.is_cuda() || pos.get_device() != r->device || pos.dim() != 1 ||
      pos.size(0) != T || !pos.is_contiguous())
    refuse("positions", "contiguous int32 [" + std::to_string(T) + "] on cuda:" + std::to_string((int)r->device), pos);
  if (T > INT32_MAX || H > INT32_MAX || D > INT32_MAX) return fail(MISAT_ERR_INVALID_ARG, "misat_rotary");
  const bool given = a[3] != Py_None;
  const at::Tensor out =
      given ? heads(a[3], "out", x.scalar_type(), r->device, T, H, D) : fresh({T, H, D}, x.scalar_type(), r->device);
  const int rc = misat_rotary(r->h, code, (int32_t)T, (int32_t)H, (int32_t)D, x.data_ptr(), x.stride(0), x.stride(1),
                              pos.data_ptr<int32_t>(), out.data_ptr(), out.stride(0), out.stride(1),
                              PyObject_IsTrue(a[4]) == 1, c10::cuda::getCurrentCUDAStream(r->device).stream());
  if (rc != MISAT_OK) return fail(rc, "misat_rotary");
  if (given) {
    written(out);
    Py_INCREF(a[3]);
    return a[3];
  }
  return THPVariable_Wrap(out);
  MISAT_END
}

bool same_heads(const Pool* p, const Batch* b) {
  if (p->hq == b->hq && p->hkv == b->hkv && p->d == b->d && p->device == b->device) return true;
  PyErr_SetString(PyExc_ValueError, "batch: made for other numbers of heads, another head_dim or another device");
  return false;
}

// (pool, batch, k, v, q or None, q_out or None) -> q_out
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 6)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  if (!b || !same_heads(p, b)) return nullptr;
  const int64_t T = b->b.n_tokens;
  const at::Tensor &k = heads(a[2], "k", p->dtype, p->device, T, p->hkv, p->d),
                   &v = heads(a[3], "v", p->dtype, p->device, T, p->hkv, p->d);
  const bool has_q = a[4] != Py_None, given = has_q && a[5] != Py_None;
  at::Tensor q, out;
  if (has_q) {
    q = heads(a[4], "q", p->dtype, p->device, T, p->hq, p->d);
    out = given ? heads(a[5], "q_out", p->dtype, p->device, T, p->hq, p->d)
                : fresh({T, p->hq, p->d}, p->dtype, p->device);
  }
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_append(p->h, &b->b, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0),
                                 v.stride(1), has_q ? q.data_ptr() : nullptr, has_q ? q.stride(0) : 0,
                                 has_q ? q.stride(1) : 0, has_q ? out.data_ptr() : nullptr, has_q ? out.stride(0) : 0,
                                 has_q ? out.stride(1) : 0, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_append");
  used(b->made, st);
  written(p->k_blocks);
  written(p->v_blocks);
  if (given) written(out);
  if (has_q && !given) return THPVariable_Wrap(out);
  PyObject* r = given ? a[5] : Py_None;
  Py_INCREF(r);
  return r;
  MISAT_END
}

// (pool, batch, q, out or None, window, return_lse) -> out or (out, lse)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 6)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  if (!b || !same_heads(p, b)) return nullptr;
  const int64_t T = b->b.n_tokens;
  const at::Tensor& q = heads(a[2], "q", p->dtype, p->device, T, p->hq, p->d);
  const bool given = a[3] != Py_None, with_lse = PyObject_IsTrue(a[5]) == 1;
  const long long window = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) return nullptr;
  const at::Tensor out =
      given ? heads(a[3], "out", p->dtype, p->device, T, p->hq, p->d) : fresh({T, p->hq, p->d}, p->dtype, p->device);
  at::Tensor lse;
  if (with_lse) lse = fresh({T, p->hq}, at::kFloat, p->device);
  if (window < 0 || window > INT32_MAX) return fail(MISAT_ERR_INVALID_ARG, "misat_kv_attend");
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_attend(p->h, &b->b, q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0),
                                 out.stride(1), with_lse ? lse.data_ptr<float>() : nullptr, (int32_t)window, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_attend");
  used(b->made, st);
  if (given) written(out);
  PyObject* o = a[3];
  if (given) Py_INCREF(o);
  else o = THPVariable_Wrap(out);
  if (!with_lse || !o) return o;
  PyObject* l = THPVariable_Wrap(lse);
  PyObject* both = l ? PyTuple_Pack(2, o, l) : nullptr;
  Py_DECREF(o);
  Py_XDECREF(l);
  return both;
  MISAT_END
}

// ---- normed heads ----

// (weight, eps, offset)
PyObject* norm_state(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 3)) return nullptr;
  const double eps = PyFloat_AsDouble(a[1]), offset = PyFloat_AsDouble(a[2]);
  if (PyErr_Occurred()) return nullptr;
  const Norm norm{tensor(a[0], "weight"), (float)eps, (float)offset};
  const at::Tensor& w = norm.w;
  if (code_of(w.scalar_type()) < 0 || !w.is_cuda() || w.dim() < 1 || w.dim() > 2)
    refuse("weight", "[head_dim] or [heads, head_dim] of bfloat16, float16 or float32 on a CUDA device", w);
  return new_state(norm);
  MISAT_END
}
// What the norm is now, for heads of d elements of a type: its weight may have been given other memory.
misat_head_norm norm_of(const Norm* norm, const char* name, at::ScalarType dtype, c10::DeviceIndex device, int64_t heads,
                        int64_t d) {
  const at::Tensor& w = norm->w;
  const bool each = w.dim() == 2;
  if ((w.scalar_type() != dtype && w.scalar_type() != at::kFloat) || !w.is_cuda() || w.get_device() != device ||
      w.dim() < 1 || w.dim() > 2 || w.size(-1) != d || (d > 1 && w.stride(-1) != 1) ||
      (each && (w.size(0) != heads || (heads > 1 && w.stride(0) < d)))) {
    std::ostringstream s;
    s << "a weight [" << d << "] or [" << heads << ", " << d << "] of " << dtype << " or float32 on cuda:" << (int)device
      << " with contiguous heads";
    refuse(name, s.str(), w);
  }
  return {w.data_ptr(), each ? (heads > 1 ? w.stride(0) : d) : 0, code_of(w.scalar_type()), norm->eps, norm->offset};
}

struct Rotation {  // the checked arguments of a call on [tokens][heads][head_dim]
  const Rope* r;
  int64_t T, H, D;
  int code;
  const int32_t* positions;
};
Rotation rotation(PyObject* rope, PyObject* ox, PyObject* positions, const char* name) {
  Rotation c{};
  c.r = state<Rope>(rope);
  if (!c.r) throw Raised{};
  const at::Tensor& x = tensor(ox, "x");
  c.code = code_of(x.scalar_type());
  if (c.code < 0 || x.dim() != 3) refuse("x", "[tokens, heads, head_dim] of bfloat16, float16 or float32", x);
  c.T = x.size(0), c.H = x.size(1), c.D = x.size(2);
  heads(ox, "x", x.scalar_type(), c.r->device, c.T, c.H, c.D);
  c.positions = ints(tensor(positions, "positions"), "positions", c.r->device, {c.T});
  if (c.T > INT32_MAX || c.H > INT32_MAX || c.D > INT32_MAX) {
    fail(MISAT_ERR_INVALID_ARG, name);
    throw Raised{};
  }
  return c;
}

// (rope, x, positions, norm, out or None) -> out
PyObject* norm_rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 5)) return nullptr;
  const Rotation c = rotation(a[0], a[1], a[2], "misat_norm_rotary");
  const Norm* norm = state<Norm>(a[3]);
  if (!norm) return nullptr;
  const at::Tensor& x = tensor(a[1], "x");
  const misat_head_norm w = norm_of(norm, "norm", x.scalar_type(), c.r->device, c.H, c.D);
  const bool given = a[4] != Py_None;
  const at::Tensor out = given ? heads(a[4], "out", x.scalar_type(), c.r->device, c.T, c.H, c.D)
                               : fresh({c.T, c.H, c.D}, x.scalar_type(), c.r->device);
  const int rc = misat_norm_rotary(c.r->h, &w, c.code, (int32_t)c.T, (int32_t)c.H, (int32_t)c.D, x.data_ptr(),
                                   x.stride(0), x.stride(1), c.positions, out.data_ptr(), out.stride(0), out.stride(1),
                                   c10::cuda::getCurrentCUDAStream(c.r->device).stream());
  if (rc != MISAT_OK) return fail(rc, "misat_norm_rotary");
  if (given) {
    written(out);
    Py_INCREF(a[4]);
    return a[4];
  }
  return THPVariable_Wrap(out);
  MISAT_END
}

PyObject* pair(PyObject* first, const at::Tensor& second) {  // takes first over
  PyObject* s = first ? THPVariable_Wrap(second) : nullptr;
  PyObject* both = s ? PyTuple_Pack(2, first, s) : nullptr;
  Py_XDECREF(first);
  Py_XDECREF(s);
  return both;
}

// (rope, x, grad, positions, norm, out or None) -> (dx, dweight)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 6)) return nullptr;
  const Rotation c = rotation(a[0], a[1], a[3], "misat_norm_rotary_backward");
  const Norm* norm = state<Norm>(a[4]);
  if (!norm) return nullptr;
  const at::Tensor& x = tensor(a[1], "x");
  const at::ScalarType dtype = x.scalar_type();
  const at::Tensor& g = heads(a[2], "grad", dtype, c.r->device, c.T, c.H, c.D);
  const misat_head_norm w = norm_of(norm, "norm", dtype, c.r->device, c.H, c.D);
  const bool given = a[5] != Py_None;
  const at::Tensor dx = given ? heads(a[5], "out", dtype, c.r->device, c.T, c.H, c.D)
                              : fresh({c.T, c.H, c.D}, dtype, c.r->device);
  int64_t bytes = 0;
  int rc = misat_norm_rotary_work(c.r->h, &w, c.code, (int32_t)c.T, (int32_t)c.H, (int32_t)c.D, &bytes);
  if (rc != MISAT_OK) return fail(rc, "misat_norm_rotary_backward");
  // Little scratch (a small call) shares the gradient's allocation.
  const at::IntArrayRef shape = norm->w.sizes();
  const int64_t own = (norm->w.numel() * 4 + 15) / 16 * 4;
  const bool together = bytes <= 64 * 1024;
  const at::Tensor work = fresh({(together ? own : 0) + bytes / 4}, at::kFloat, c.r->device);
  const at::Tensor dw = together ? piece(work, 0, shape, norm->w.scalar_type())
                                 : fresh(shape, norm->w.scalar_type(), c.r->device);
  float* const scratch = work.data_ptr<float>() + (together ? own : 0);
  rc = misat_norm_rotary_backward(c.r->h, &w, c.code, (int32_t)c.T, (int32_t)c.H, (int32_t)c.D, x.data_ptr(),
                                  x.stride(0), x.stride(1), g.data_ptr(), g.stride(0), g.stride(1), c.positions,
                                  dx.data_ptr(), dx.stride(0), dx.stride(1), dw.data_ptr(), c.D, scratch, bytes,
                                  c10::cuda::getCurrentCUDAStream(c.r->device).stream());
  if (rc != MISAT_OK) return fail(rc, "misat_norm_rotary_backward");
  PyObject* o = a[5];
  if (given) {
    written(dx);
    Py_INCREF(o);
  } else {
    o = THPVariable_Wrap(dx);
  }
  return pair(o, dw);
  MISAT_END
}

// ---- trees of drafted tokens ----

// The tree was made for this batch's tokens.
bool same_tokens(const Tree* t, const Batch* b) {
  if (t->n_tokens == b->b.n_tokens && t->max_q == b->b.max_q && t->device == b->device) return true;
  PyErr_SetString(PyExc_ValueError, "tree: made for a batch of other tokens or another device");
  return false;
}

// (pool, batch, k, v, q or None, q_out or None, q_norm or None, k_norm or None, tree or None) -> q_out
PyObject* append_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 9)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  if (!b || !same_heads(p, b)) return nullptr;
  const int64_t T = b->b.n_tokens;
  const at::Tensor &k = heads(a[2], "k", p->dtype, p->device, T, p->hkv, p->d),
                   &v = heads(a[3], "v", p->dtype, p->device, T, p->hkv, p->d);
  const bool has_q = a[4] != Py_None, given = has_q && a[5] != Py_None;
  at::Tensor q, out;
  if (has_q) {
    q = heads(a[4], "q", p->dtype, p->device, T, p->hq, p->d);
    out = given ? heads(a[5], "q_out", p->dtype, p->device, T, p->hq, p->d)
                : fresh({T, p->hq, p->d}, p->dtype, p->device);
  }
  misat_head_norm norms[2];
  const misat_head_norm* norm[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i) {
    if (a[6 + i] == Py_None) continue;
    const Norm* w = state<Norm>(a[6 + i]);
    if (!w) return nullptr;
    norms[i] = norm_of(w, i ? "k_norm" : "q_norm", p->dtype, p->device, i ? p->hkv : p->hq, p->d);
    norm[i] = norms + i;
  }
  const Tree* t = a[8] == Py_None ? nullptr : state<Tree>(a[8]);
  if (a[8] != Py_None && (!t || !same_tokens(t, b))) return nullptr;
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_append_norm(
      p->h, &b->b, norm[0], norm[1], t ? &t->d : nullptr, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
      v.stride(0), v.stride(1), has_q ? q.data_ptr() : nullptr, has_q ? q.stride(0) : 0, has_q ? q.stride(1) : 0,
      has_q ? out.data_ptr() : nullptr, has_q ? out.stride(0) : 0, has_q ? out.stride(1) : 0, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_append_norm");
  used(b->made, st);
  if (t) used(t->made, st);
  written(p->k_blocks);
  written(p->v_blocks);
  if (given) written(out);
  if (has_q && !given) return THPVariable_Wrap(out);
  PyObject* r = given ? a[5] : Py_None;
  Py_INCREF(r);
  return r;
  MISAT_END
}

// (pool, batch, parents, window) -> (depth, bits, tree)
PyObject* tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 4)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  if (!b || !same_heads(p, b)) return nullptr;
  const int64_t T = b->b.n_tokens;
  const int32_t* parents = ints(tensor(a[2], "parents"), "parents", p->device, {T});
  const int32_t window = int32_of(a[3], "window");
  if (window < 0 || b->b.max_q > MISAT_KV_TREE_NODES) return fail(MISAT_ERR_INVALID_ARG, "misat_kv_tree");
  const int32_t words = (b->b.max_q + 31) / 32;
  const at::Tensor all_words = fresh({T * (words + 1)}, at::kInt, p->device), depth = piece(all_words, T * words, {T}),
                   bits = piece(all_words, 0, {T, words});
  Tree t{{depth.data_ptr<int32_t>(), reinterpret_cast<uint32_t*>(bits.data_ptr<int32_t>()), words, window},
         T, b->b.max_q, p->device, {nullptr, {depth, bits}}};
  t.made.on = ordered(p);
  const int rc = misat_kv_tree(p->h, &b->b, parents, window, const_cast<int32_t*>(t.d.depth),
                               const_cast<uint32_t*>(t.d.bits), words, t.made.on);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_tree");
  used(b->made, t.made.on);
  PyObject* c = new_state(t);
  if (!c) return nullptr;
  PyObject *d = THPVariable_Wrap(depth), *w = d ? THPVariable_Wrap(bits) : nullptr;
  PyObject* all = w ? PyTuple_Pack(3, d, w, c) : nullptr;
  Py_DECREF(c);
  Py_XDECREF(d);
  Py_XDECREF(w);
  return all;
  MISAT_END
}

// (pool, batch, q, out or None, tree, return_lse) -> out or (out, lse)
PyObject* attend_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 6)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  const Tree* t = b ? state<Tree>(a[4]) : nullptr;
  if (!t || !same_heads(p, b) || !same_tokens(t, b)) return nullptr;
  const int64_t T = b->b.n_tokens;
  const at::Tensor& q = heads(a[2], "q", p->dtype, p->device, T, p->hq, p->d);
  const bool given = a[3] != Py_None, with_lse = PyObject_IsTrue(a[5]) == 1;
  const at::Tensor out =
      given ? heads(a[3], "out", p->dtype, p->device, T, p->hq, p->d) : fresh({T, p->hq, p->d}, p->dtype, p->device);
  at::Tensor lse;
  if (with_lse) lse = fresh({T, p->hq}, at::kFloat, p->device);
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_attend_tree(p->h, &b->b, &t->d, q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(),
                                      out.stride(0), out.stride(1), with_lse ? lse.data_ptr<float>() : nullptr, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_attend_tree");
  used(b->made, st);
  used(t->made, st);
  PyObject* o = a[3];
  if (given) {
    written(out);
    Py_INCREF(o);
  } else {
    o = THPVariable_Wrap(out);
  }
  return with_lse ? pair(o, lse) : o;
  MISAT_END
}

// (pool, batch, path, n_keep, out or None) -> kv_len
PyObject* keep(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 5)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  const Batch* b = p ? state<Batch>(a[1]) : nullptr;
  if (!b || !same_heads(p, b)) return nullptr;
  const int64_t seqs = b->b.n;
  const at::Tensor& path = tensor(a[2], "path");
  const int64_t width = path.dim() == 2 ? path.size(1) : 0;
  const int32_t* nodes = ints(path, "path", p->device, {seqs, width});
  const int32_t* many = ints(tensor(a[3], "n_keep"), "n_keep", p->device, {seqs});
  const bool given = a[4] != Py_None;
  const at::Tensor out = given ? tensor(a[4], "out") : fresh({seqs}, at::kInt, p->device);
  int32_t* len = ints(out, "out", p->device, {seqs});
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_keep(p->h, &b->b, nodes, width, many, len, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_keep");
  used(b->made, st);
  written(p->k_blocks);
  written(p->v_blocks);
  if (!given) return THPVariable_Wrap(out);
  written(out);
  Py_INCREF(a[4]);
  return a[4];
  MISAT_END
}

// (pool, block_table, ring, state, new, kv_len, shared or None, n_tokens, max_q, out or None)
//   -> (state, q_off, kv_len, positions, slots, batch)
PyObject* tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MISAT_TRY
  if (!count(n, 10)) return nullptr;
  Pool* p = state<Pool>(a[0]);
  if (!p) return nullptr;
  const at::Tensor &table = tensor(a[1], "block_table"), &ring = tensor(a[2], "ring"), &fresh_tokens = tensor(a[4], "new");
  const int64_t seqs = fresh_tokens.dim() == 1 ? fresh_tokens.size(0) : 0;
  misat_kv_step s{};
  s.new_tokens = ints(fresh_tokens, "new", p->device, {seqs});
  s.kv_len = ints(tensor(a[5], "kv_len"), "kv_len", p->device, {seqs});
  if (a[6] != Py_None) s.shared = ints(tensor(a[6], "shared"), "shared", p->device, {seqs});
  const at::Tensor& before = tensor(a[3], "state");
  s.state = ints(before, "state", p->device, {seqs + 2});
  const int64_t columns = table_columns(table, p->device, seqs, s.table_stride);
  const int64_t places = ring.dim() == 1 ? ring.size(0) : 0;
  s.ring = ints(ring, "ring", p->device, {places});
  s.block_table = table.data_ptr<int32_t>();
  s.n_tokens = int32_of(a[7], "n_tokens");
  s.max_q = int32_of(a[8], "max_q");
  if (seqs > INT32_MAX || columns > INT32_MAX || places > INT32_MAX || s.n_tokens < 0 || s.n_tokens > INT32_MAX - 4096)
    return fail(MISAT_ERR_INVALID_ARG, "misat_kv_tables");
  s.n = (int32_t)seqs;
  s.columns = (int32_t)columns;
  s.ring_size = (int32_t)places;
  const bool given = a[9] != Py_None;
  // One allocation for what there is of each sequence, each array at a 16-byte boundary, and one for the tokens'.
  const int64_t bytes = MISAT_KV_TABLES_WORK(seqs), row = (seqs + 2 + 3) / 4 * 4;
  const at::Tensor rows = fresh({3 * row + bytes / 4}, at::kInt, p->device);
  const int64_t T = s.n_tokens, half = (T + 1) / 2;
  const at::Tensor after = given ? tensor(a[9], "out") : piece(rows, 0, {seqs + 2}), q_off = piece(rows, row, {seqs + 1}),
                   len = piece(rows, 2 * row, {seqs}), tokens = fresh({T + half}, at::kLong, p->device),
                   slots = piece(tokens, 0, {T}, at::kLong), positions = piece(tokens, 2 * T, {T});
  s.state_out = ints(after, "out", p->device, {seqs + 2});
  s.q_off = q_off.data_ptr<int32_t>();
  s.kv_len_out = len.data_ptr<int32_t>();
  s.positions = positions.data_ptr<int32_t>();
  s.slots = slots.data_ptr<int64_t>();
  const cudaStream_t st = ordered(p);
  const int rc = misat_kv_tables(p->h, &s, rows.data_ptr<int32_t>() + 3 * row, bytes, st);
  if (rc != MISAT_OK) return fail(rc, "misat_kv_tables");
  written(table);
  written(ring);
  if (given) written(after);
  const Batch b{{s.n, s.n_tokens, s.max_q, s.q_off, s.kv_len_out, s.block_table, s.table_stride},
                p->hq, p->hkv, p->d, p->device, {st, {q_off, len}}};
  PyObject* all = PyTuple_New(6);
  if (!all) return nullptr;
  PyObject* first = a[9];
  if (given) Py_INCREF(first);
  else first = THPVariable_Wrap(after);
  PyObject* items[6] = {first, THPVariable_Wrap(q_off), THPVariable_Wrap(len), THPVariable_Wrap(positions),
                        THPVariable_Wrap(slots), new_state(b)};
  bool ok = true;
  for (int i = 0; i < 6; ++i) {
    ok = ok && items[i];
    PyTuple_SET_ITEM(all, i, items[i]);
  }
  if (ok) return all;
  Py_DECREF(all);
  return nullptr;
  MISAT_END
}

// (pool): waits, and raises the pool's sticky device error
PyObject* sync(PyObject*, PyObject* c) {
  MISAT_TRY
  Pool* p = state<Pool>(c);
  if (!p) return nullptr;
  const cudaStream_t st = ordered(p);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = misat_kv_sync(p->h, st);
  Py_END_ALLOW_THREADS
  if (rc != MISAT_OK) return fail(rc, "misat_kv_sync");
  Py_RETURN_NONE;
  MISAT_END
}

#define MISAT_FAST(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", init, METH_O, nullptr},
                         MISAT_FAST(rope_state),
                         MISAT_FAST(pool_state),
                         MISAT_FAST(batch_state),
                         MISAT_FAST(rotary),
                         MISAT_FAST(append),
                         MISAT_FAST(attend),
                         MISAT_FAST(norm_state),
                         MISAT_FAST(norm_rotate),
                         MISAT_FAST(norm_backward),
                         MISAT_FAST(append_norm),
                         MISAT_FAST(tree),
                         MISAT_FAST(attend_tree),
                         MISAT_FAST(keep),
                         MISAT_FAST(tables),
                         {"sync", sync, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
