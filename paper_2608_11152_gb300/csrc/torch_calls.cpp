// The KV operators' calls on torch tensors: checks of the arguments, the result's memory, the current
// stream, and the C entry point, in one step.
//
// These calls are made once a layer and token.  Through ctypes the same steps took 9 us of a call whose
// kernel takes 3 (torch.empty 3.3, checks and attribute reads 1.8, argument conversion 1.5, launch 2.1).
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>

#include "../../include/misat.h"

namespace {

PyObject* g_error = nullptr;  // MisatError

struct Rope {
  misat_rope* h;
  c10::DeviceIndex device;
};
struct Pool {
  misat_kv* h;
  c10::DeviceIndex device;
  at::Tensor k_blocks, v_blocks;
  at::ScalarType dtype;
  int64_t hq, hkv, d;
  cudaStream_t last;  // of the last call outside a capture
  bool called;
};
struct Batch {
  misat_kv_batch b;
  int64_t hq, hkv, d;
  c10::DeviceIndex device;
};

template <class S>
void free_state(PyObject* c) {
  delete static_cast<S*>(PyCapsule_GetPointer(c, nullptr));
}
template <class S>
PyObject* new_state(const S& s) {
  S* p = new S(s);
  PyObject* c = PyCapsule_New(p, nullptr, free_state<S>);
  if (!c) delete p;
  return c;
}
template <class S>
S* state(PyObject* c) {
  return static_cast<S*>(PyCapsule_GetPointer(c, nullptr));
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
// Autograd finds out by its version that a tensor it has saved was written.
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
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
  const int64_t seqs = len.dim() == 1 ? len.size(0) : -1;
  auto ints = [&](const at::Tensor& t, const char* name, int64_t size) {
    if (t.scalar_type() != at::kInt || !t.is_cuda() || t.get_device() != p->device || t.dim() != 1 || size < 0 ||
        t.size(0) != size || !t.is_contiguous())
      refuse(name, "contiguous int32 [" + std::to_string(size) + "] on cuda:" + std::to_string((int)p->device), t);
  };
  ints(len, "kv_len", seqs);
  ints(off, "q_off", seqs + 1);
  const bool shaped = table.scalar_type() == at::kInt && table.is_cuda() && table.get_device() == p->device &&
                      table.dim() == 2 && table.size(0) == seqs;
  const int64_t blocks = shaped ? table.size(1) : 0, stride = shaped && seqs > 1 ? table.stride(0) : blocks;
  if (!shaped || (blocks > 1 && table.stride(1) != 1) || stride < blocks)
    refuse("block_table",
           "int32 [" + std::to_string(seqs) + ", blocks] on cuda:" + std::to_string((int)p->device) +
               " with contiguous rows that do not overlap",
           table);
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
  const int rc = misat_kv_append(p->h, &b->b, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0),
                                 v.stride(1), has_q ? q.data_ptr() : nullptr, has_q ? q.stride(0) : 0,
                                 has_q ? q.stride(1) : 0, has_q ? out.data_ptr() : nullptr, has_q ? out.stride(0) : 0,
                                 has_q ? out.stride(1) : 0, ordered(p));
  if (rc != MISAT_OK) return fail(rc, "misat_kv_append");
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
  const int rc =
      window < 0 || window > INT32_MAX
          ? MISAT_ERR_INVALID_ARG
          : misat_kv_attend(p->h, &b->b, q.data_ptr(), q.stride(0), q.stride(1), out.data_ptr(), out.stride(0),
                            out.stride(1), with_lse ? lse.data_ptr<float>() : nullptr, (int32_t)window, ordered(p));
  if (rc != MISAT_OK) return fail(rc, "misat_kv_attend");
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
                         {"sync", sync, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
