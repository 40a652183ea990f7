// Native marshalling of the calls that a program makes per layer.  A small layer's call costs the host more than the device
// (one image through a 384 x 384 projection: 3.8 us of kernel, 7.3 us per call in Python), so a call whose arguments are all
// in the ordinary form -- plain device tensors of the right types and shapes, Python integers -- is read, checked and
// handed to the C ABI here.  Anything else is declined (NotImplemented), and the Python function goes on with it: it
// knows the other forms that are accepted and names what is wrong with the ones that are not.  Nothing is kept
// between calls.
// Measured per call: the projection above 7.3 -> 4.1 us; 768 -> 1000 at 4:8 on 8 tokens, plain, 8.2 -> 6.2 (5.0 with a kernel
// that has become faster since); the twelve calls and sixteen allocations that compress a block by scores and expand it 94 -> 63. The training
// products and the int8 layer on small operands: dX in one launch 7.2 -> 4.0 us (in two, with scratch of the call's own, 7.5 to 8.0), dW
// in two launches 11 -> 8, a prepared int8 call 7.5 -> 3.6; a plain call, whose scratch is looked up in the table that Python keeps,
// 4.0 -> 3.5.  (A launch alone takes the host 3.0 to 3.5; all of these vary by a quarter from host to host.)
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cmath>
#include <exception>
#include <optional>
#include <vector>

#include "nm_sparse.h"

namespace {

// The C ABI of the library that Python has loaded (set once by bind), and the Python helpers of the rare ways on.
struct Library {
  decltype(&nm_prune) prune;
  decltype(&nm_prune_scored) prune_scored;
  decltype(&nm_pack) pack;
  decltype(&nm_unpack) unpack;
  decltype(&nm_linear_forward) forward;
  decltype(&nm_linear_forward_prepared) forward_prepared;
  decltype(&nm_linear_forward_static) forward_static;
  decltype(&nm_spmm_workspace_bytes) workspace_bytes;
  decltype(&nm_values_bytes) values_bytes;
  decltype(&nm_index_bytes) index_bytes;
  // may be missing: a prepared layer is then multiplied uncut
  decltype(&nm_linear_forward_prepared_scratch) forward_prepared_scratch;
  decltype(&nm_prepared_scratch_bytes) prepared_scratch_bytes;
  // may be missing: those calls are then declined
  decltype(&nm_linear_backward_input) backward_input;
  decltype(&nm_linear_backward_weight) backward_weight;
  decltype(&nm_linear_backward_input_scratch) backward_input_scratch;
  decltype(&nm_backward_input_workspace_bytes) backward_input_bytes;
  decltype(&nm_backward_input_scratch_bytes) backward_input_scratch_bytes;
  decltype(&nm_backward_input_scratch_pays) backward_input_scratch_pays;
  decltype(&nm_linear_backward_weight_scratch) backward_weight_scratch;
  decltype(&nm_backward_weight_scratch_bytes) backward_weight_scratch_bytes;
  decltype(&nm_linear_forward_i8) i8;
  decltype(&nm_linear_forward_i8_prepared) i8_prepared;
  decltype(&nm_linear_forward_i8_packed) i8_packed;
  decltype(&nm_linear_forward_i8_packed_prepared) i8_packed_prepared;
  decltype(&nm_i8_workspace_bytes) i8_bytes;
  decltype(&nm_layer_norm) layer_norm;
  decltype(&nm_layer_norm_backward) layer_norm_backward;
  decltype(&nm_layer_norm_backward_workspace_bytes) layer_norm_backward_bytes;
  decltype(&nm_rotary) rotary;
  decltype(&nm_attention) attention;
  decltype(&nm_attention_workspace_bytes) attention_bytes;
  decltype(&nm_attention_backward) attention_backward;
  decltype(&nm_attention_backward_workspace_bytes) attention_backward_bytes;
  decltype(&nm_head_norm) head_norm;
  decltype(&nm_head_norm_backward) head_norm_backward;
  decltype(&nm_head_norm_backward_workspace_bytes) head_norm_backward_bytes;
  decltype(&nm_cache_write) cache_write;
  decltype(&nm_cache_read) cache_read;
  decltype(&nm_attention_paged) attention_paged;
  decltype(&nm_attention_paged_workspace_bytes) attention_paged_bytes;
} lib;
PyObject* raise_status;    // raises NmError for a status that is not NM_OK
PyObject* find_workspace;  // the scratch tensor of a device and stream
PyObject* workspaces;      // where find_workspace keeps them: (device type, index, stream) -> tensor; may be missing

PyObject* declined() { Py_RETURN_NOTIMPLEMENTED; }

// A device tensor that is nothing but that: no subclass, no functional transform's wrapper, no lazy conjugate or negation.
bool plain(PyObject* obj, at::ScalarType type, const at::Tensor** out) {
  if (!THPVariable_CheckExact(obj)) return false;
  const at::Tensor& t = THPVariable_Unpack(obj);
  constexpr c10::DispatchKeySet ordinary({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView,
                                          c10::DispatchKey::AutocastCUDA});
  if (!t.defined() || t.key_set() - ordinary != c10::DispatchKeySet(c10::BackendComponent::CUDABit) || t.scalar_type() != type ||
      !t.has_storage())
    return false;
  *out = &t;
  return true;
}

bool integer(PyObject* obj, int64_t lo, int64_t hi, int64_t* out) {
  if (!PyLong_CheckExact(obj)) return false;
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(obj, &overflow);
  if (overflow || v < lo || v > hi) return false;
  *out = v;
  return true;
}
bool level(PyObject* n, PyObject* m, int32_t* N, int32_t* M) {
  int64_t a, b;
  if (!integer(n, 0, 16, &a) || !integer(m, 0, 16, &b)) return false;
  *N = (int32_t)a;
  *M = (int32_t)b;
  return true;
}

// rows, columns and leading dimension of a matrix whose rows are contiguous
struct Matrix { int64_t rows, cols, ld; };
bool matrix(const at::Tensor& t, Matrix* m) {
  if (t.dim() != 2) return false;
  m->rows = t.size(0);
  m->cols = t.size(1);
  if (t.stride(1) != 1 && m->cols > 1) return false;
  m->ld = m->rows > 1 ? t.stride(0) : m->cols;
  return true;
}
bool whole(const at::Tensor& t) { return t.dim() == 2 && t.is_contiguous(); }

// The stream of a call: the given one, or the current one of the current device.
bool stream_of(PyObject* obj, void** out) {
  if (obj == Py_None) {
    *out = c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream();
    return true;
  }
  PyObject* handle = PyObject_GetAttrString(obj, "cuda_stream");
  if (handle == nullptr) { PyErr_Clear(); return false; }
  const bool ok = PyLong_CheckExact(handle);
  if (ok) *out = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (PyErr_Occurred()) { PyErr_Clear(); return false; }
  return ok;
}

// Tracing modes and the like see every tensor operation: they get the Python functions.
bool observed() { return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set(); }

template <class T>
T* pointer(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

// f without the interpreter lock: other threads run meanwhile, and a stream's host function that needs it can end.  f allocates
// the outputs, which may free cached memory and wait for the device, and calls the library; the arguments' pointers are taken
// before.  (One release for both: each takes 0.1 us.)  An exception of f goes on when the lock is held again.  Not noexcept: where
// the interpreter has ended meanwhile, taking its lock again ends this thread by unwinding its stack.
template <class F>
auto unlocked(F&& f) {
  std::optional<decltype(f())> r;
  std::exception_ptr failed;
  PyThreadState* self = PyEval_SaveThread();
  try {
    r.emplace(f());
  } catch (...) {
    failed = std::current_exception();
  }
  PyEval_RestoreThread(self);
  if (failed) std::rethrow_exception(failed);
  return *std::move(r);
}
PyObject* result(int32_t st, PyObject* value) {  // steals value
  if (st == NM_OK) return value;
  Py_XDECREF(value);
  PyObject* r = PyObject_CallFunction(raise_status, "i", (int)st);
  Py_XDECREF(r);
  return nullptr;
}

at::Tensor fresh(at::Device device, int64_t rows, int64_t cols, at::ScalarType type) {
  return at::empty({rows, cols}, at::TensorOptions().dtype(type).device(device));
}

// Bytes that go to later work of this stream only, and back to it when the call has been issued.  Taken from the allocator without a
// tensor around them.
struct Scratch {
  void* ptr;
  Scratch(void* s, at::Device device, size_t bytes) {
    const c10::DeviceIndex current = c10::hip::current_device();
    c10::OptionalDeviceGuard on;
    if (device.index() != current && s != c10::hip::getCurrentHIPStream(current).stream()) on.reset_device(device);
    ptr = c10::hip::HIPCachingAllocator::raw_alloc_with_stream(bytes, static_cast<hipStream_t>(s));
  }
  Scratch(const Scratch&) = delete;
  ~Scratch() { c10::hip::HIPCachingAllocator::raw_delete(ptr); }
};

// Whether memory allocated now, on the current device, goes to later work of this stream only.
bool on_current_stream(void* s, at::Device* here) {
  *here = at::Device(at::kCUDA, c10::hip::current_device());
  return s == c10::hip::getCurrentHIPStream(here->index()).stream();
}

// The workspace of a call: the given tensor, or the scratch of its device and stream, held until the call has returned.
struct Workspace {
  THPObjectPtr found;
  void* ptr = nullptr;
  size_t bytes = 0;
};
enum Take { TAKEN, DECLINED, FAILED };
Take given_workspace(PyObject* given, Workspace* w) {
  if (given == Py_None) return TAKEN;
  const at::Tensor* ws = nullptr;
  if (!THPVariable_CheckExact(given) || !(ws = &THPVariable_Unpack(given))->is_cuda() || !ws->has_storage()) return DECLINED;
  w->ptr = ws->data_ptr();
  w->bytes = ws->nbytes();
  return TAKEN;
}
// `like`: the tensor on whose device it lies (asking Python for it takes 0.7 us, reading its table 0.1)
Take scratch_workspace(size_t need, PyObject* like, PyObject* stream, void* s, Workspace* w) {
  if (workspaces != nullptr) {
    THPObjectPtr key(Py_BuildValue("(snK)", "cuda", (Py_ssize_t)THPVariable_Unpack(like).device().index(), (unsigned long long)(uintptr_t)s));
    if (!key) return FAILED;
    PyObject* kept = PyDict_GetItemWithError(workspaces, key.get());
    if (kept == nullptr && PyErr_Occurred()) return FAILED;
    if (kept != nullptr) {
      Py_INCREF(kept);
      w->found = THPObjectPtr(kept);
      if (given_workspace(kept, w) == TAKEN && w->bytes >= need) return TAKEN;
    }
  }
  THPObjectPtr device(PyObject_GetAttrString(like, "device"));
  if (!device) return FAILED;
  w->found = THPObjectPtr(PyObject_CallFunction(find_workspace, "nOO", (Py_ssize_t)need, device.get(), stream));
  return w->found ? given_workspace(w->found.get(), w) : FAILED;
}

// The output of a call: `given` (out), or made on the device of its operands in the type asked for (out_dtype).
struct Output {
  PyObject* given;
  at::Tensor made;
  at::ScalarType type;
  int64_t rows, cols, ld;
  void* ptr;
  int32_t code;
  bool read(PyObject* dtype, PyObject* out, int64_t r, int64_t c, bool i32) {
    given = out;
    rows = r;
    cols = c;
    type = at::kFloat;
    if (out != Py_None) {
      const at::Tensor* t = nullptr;
      Matrix m;
      if (!plain(out, at::kBFloat16, &t) && !plain(out, at::kFloat, &t) && !(i32 && plain(out, at::kInt, &t))) return false;
      if (!matrix(*t, &m) || m.rows != r || m.cols != c) return false;
      type = t->scalar_type();
      ld = m.ld;
      ptr = t->data_ptr();
    } else if (dtype != Py_None) {
      if (!THPDtype_Check(dtype)) return false;
      type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    }
    if (type == at::kFloat) code = NM_OUT_F32;
    else if (type == at::kBFloat16) code = NM_OUT_BF16;
    else if (i32 && type == at::kInt) code = NM_OUT_I32;
    else return false;
    return true;
  }
  void make(at::Device device) {  // (without the interpreter lock)
    if (given != Py_None) return;
    made = fresh(device, rows, cols, type);
    ptr = made.data_ptr();
    ld = cols;
  }
  PyObject* take() {
    if (given == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
  }
};

// prune(W, N, M, W_masked, stream)
PyObject* prune(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *W, *Wm = nullptr;
  Matrix w, wm;
  int32_t N, M;
  void* s;
  if (n != 5 || observed() || !plain(a[0], at::kBFloat16, &W) || !matrix(*W, &w) || !level(a[1], a[2], &N, &M)) return declined();
  if (a[3] != Py_None &&
      (!plain(a[3], at::kBFloat16, &Wm) || !matrix(*Wm, &wm) || wm.rows != w.rows || wm.cols != w.cols || wm.ld != w.ld))
    return declined();
  if (!stream_of(a[4], &s)) return declined();
  at::Tensor mask;
  const at::Device device = W->device();
  const uint16_t* wp = pointer<uint16_t>(W);
  uint16_t* wmp = pointer<uint16_t>(Wm);
  const int32_t st = unlocked([&] {
    mask = fresh(device, w.rows, (w.cols + 31) / 32, at::kInt);
    return lib.prune(wp, w.rows, w.cols, w.ld, N, M, pointer<uint32_t>(&mask), wmp, s);
  });
  return result(st, THPVariable_Wrap(std::move(mask)));
  END_HANDLE_TH_ERRORS
}

// prune_scored(score, N, M, stream)
PyObject* prune_scored(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* score;
  Matrix m;
  int32_t N, M;
  void* s;
  if (n != 4 || observed() || !plain(a[0], at::kFloat, &score) || !matrix(*score, &m) || !level(a[1], a[2], &N, &M) ||
      !stream_of(a[3], &s))
    return declined();
  at::Tensor mask;
  const at::Device device = score->device();
  const float* sp = pointer<float>(score);
  const int32_t st = unlocked([&] {
    mask = fresh(device, m.rows, (m.cols + 31) / 32, at::kInt);
    return lib.prune_scored(sp, m.rows, m.cols, m.ld, N, M, pointer<uint32_t>(&mask), s);
  });
  return result(st, THPVariable_Wrap(std::move(mask)));
  END_HANDLE_TH_ERRORS
}

// pack(W, N, M, mask, stream)
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *W, *mask = nullptr;
  Matrix w;
  int32_t N, M;
  void* s;
  if (n != 5 || observed() || !plain(a[0], at::kBFloat16, &W) || !matrix(*W, &w) || w.rows < 1 || !level(a[1], a[2], &N, &M))
    return declined();
  if (a[3] != Py_None && (!plain(a[3], at::kInt, &mask) || !whole(*mask) || mask->size(0) != w.rows || mask->size(1) != (w.cols + 31) / 32))
    return declined();
  const size_t vb = lib.values_bytes(w.rows, w.cols, N, M);
  if (vb == 0 || !stream_of(a[4], &s)) return declined();
  at::Tensor values, indices;
  const at::Device device = W->device();
  const uint16_t* wp = pointer<uint16_t>(W);
  const uint32_t* mp = pointer<uint32_t>(mask);
  const int32_t st = unlocked([&] {
    values = fresh(device, w.rows, (int64_t)vb / (2 * w.rows), at::kBFloat16);
    indices = fresh(device, w.rows, (int64_t)lib.index_bytes(w.rows, w.cols, N, M) / (4 * w.rows), at::kInt);
    return lib.pack(wp, w.rows, w.cols, w.ld, N, M, mp, pointer<uint16_t>(&values), pointer<uint32_t>(&indices), s);
  });
  return result(st, Py_BuildValue("(NN)", THPVariable_Wrap(std::move(values)), THPVariable_Wrap(std::move(indices))));
  END_HANDLE_TH_ERRORS
}

// unpack(values, indices, K, N, M, stream)
PyObject* unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *values, *indices;
  int64_t K;
  int32_t N, M;
  void* s;
  if (n != 6 || observed() || !plain(a[0], at::kBFloat16, &values) || !whole(*values) || !plain(a[1], at::kInt, &indices) ||
      !whole(*indices) || !integer(a[2], 1, 1ll << 40, &K) || !level(a[3], a[4], &N, &M) || !stream_of(a[5], &s))
    return declined();
  const int64_t O = values->size(0);
  at::Tensor Wd;
  const at::Device device = values->device();
  const uint16_t* vp = pointer<uint16_t>(values);
  const uint32_t* ip = pointer<uint32_t>(indices);
  const int32_t st = unlocked([&] {
    Wd = fresh(device, O, K, at::kBFloat16);
    return lib.unpack(vp, ip, O, K, N, M, pointer<uint16_t>(&Wd), K, s);
  });
  return result(st, THPVariable_Wrap(std::move(Wd)));
  END_HANDLE_TH_ERRORS
}

// forward(values, indices, K, N, M, X, bias, out_dtype, out, workspace, stream, how); how: 0 plain, 1 prepared, 2 straight
// from the packed format, 3 on the library's fixed scratch
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *values, *indices, *X, *bias = nullptr, *out = nullptr;
  int64_t K, how;
  int32_t N, M;
  Matrix x, y;
  void* s;
  if (n != 12 || observed() || !plain(a[0], at::kBFloat16, &values) || !whole(*values) || !plain(a[1], at::kInt, &indices) ||
      !whole(*indices) || !integer(a[2], 1, 1ll << 40, &K) || !level(a[3], a[4], &N, &M) || !plain(a[5], at::kBFloat16, &X) ||
      !matrix(*X, &x) || x.cols != K || !integer(a[11], 0, 3, &how))
    return declined();
  const int64_t O = values->size(0), T = x.rows;
  if (a[6] != Py_None && (!plain(a[6], at::kFloat, &bias) || bias->numel() != O || !bias->is_contiguous())) return declined();
  int32_t code;
  at::Tensor made;
  if (a[8] != Py_None) {
    if (plain(a[8], at::kBFloat16, &out)) code = NM_OUT_BF16;
    else if (plain(a[8], at::kFloat, &out)) code = NM_OUT_F32;
    else return declined();
    if (!matrix(*out, &y) || y.rows != T || y.cols != O) return declined();
  } else {
    at::ScalarType type = at::kFloat;
    if (a[7] != Py_None) {
      if (!THPDtype_Check(a[7])) return declined();
      type = reinterpret_cast<THPDtype*>(a[7])->scalar_type;
      if (type != at::kFloat && type != at::kBFloat16) return declined();
    }
    code = type == at::kFloat ? NM_OUT_F32 : NM_OUT_BF16;
  }
  if (!stream_of(a[10], &s)) return declined();
  Workspace ws;
  if (how != 3) {
    if (a[9] == Py_None && how != 2) {
      const size_t need = lib.workspace_bytes(O, K, N, M, T);
      if (need != 0 && how == 1) return declined();  // (refused, or a ragged reduction without its copy)
      if (need != 0)
        if (const Take t = scratch_workspace(need, a[5], a[10], s, &ws); t != TAKEN) return t == DECLINED ? declined() : nullptr;
    } else if (given_workspace(a[9], &ws) != TAKEN) {
      return declined();
    }
  }
  void* const ws_ptr = ws.ptr;
  const size_t ws_bytes = ws.bytes;
  // partial sums of a prepared layer that is cut along K: scratch of the call, allocated on its stream, so that the memory goes to
  // later work of that stream only.  (Not for a workspace of the operand part alone, which asks for the uncut product.)
  size_t scratch_bytes = how == 1 && lib.prepared_scratch_bytes ? lib.prepared_scratch_bytes(O, K, N, M, T) : 0;
  if (scratch_bytes != 0 && ws_bytes < lib.workspace_bytes(O, K, N, M, T)) scratch_bytes = 0;
  at::Device here = X->device();
  if (scratch_bytes != 0 && !on_current_stream(s, &here)) return declined();
  const uint16_t *v = pointer<uint16_t>(values), *xp = pointer<uint16_t>(X);
  const uint32_t* ix = pointer<uint32_t>(indices);
  const float* b = pointer<float>(bias);
  void* yp = pointer<void>(out);
  const at::Device device = X->device();
  const int32_t st = unlocked([&] {
    if (out == nullptr) {
      made = fresh(device, T, O, code == NM_OUT_F32 ? at::kFloat : at::kBFloat16);
      yp = made.data_ptr();
      y.ld = O;
    }
    if (how == 3) return lib.forward_static(v, ix, O, K, N, M, xp, T, x.ld, b, yp, y.ld, code, s);
    if (scratch_bytes != 0) {
      const at::Tensor scratch = fresh(here, 1, (int64_t)scratch_bytes, at::kByte);
      return lib.forward_prepared_scratch(v, ix, O, K, N, M, xp, T, x.ld, b, yp, y.ld, code, ws_ptr, ws_bytes,
                                          scratch.data_ptr(), scratch_bytes, s);
    }
    if (how == 1) return lib.forward_prepared(v, ix, O, K, N, M, xp, T, x.ld, b, yp, y.ld, code, ws_ptr, ws_bytes, s);
    return lib.forward(v, ix, O, K, N, M, xp, T, x.ld, b, yp, y.ld, code, ws_ptr, ws_bytes, s);
  });
  if (out != nullptr) {
    Py_INCREF(a[8]);
    return result(st, a[8]);
  }
  return result(st, THPVariable_Wrap(std::move(made)));
  END_HANDLE_TH_ERRORS
}

// backward_input(Ws, dY, out_dtype, out, workspace, stream)
PyObject* backward_input(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *W, *dY;
  Matrix w, dy;
  Output y;
  void* s;
  if (n != 6 || lib.backward_input == nullptr || lib.backward_input_scratch == nullptr || lib.backward_input_bytes == nullptr ||
      lib.backward_input_scratch_bytes == nullptr || lib.backward_input_scratch_pays == nullptr || observed() || !plain(a[0], at::kBFloat16, &W) ||
      !matrix(*W, &w) || !plain(a[1], at::kBFloat16, &dY) || !matrix(*dY, &dy) || dy.cols != w.rows ||
      !y.read(a[2], a[3], dy.rows, w.cols, false) || !stream_of(a[5], &s))
    return declined();
  Workspace ws;
  const size_t need = a[4] == Py_None ? lib.backward_input_bytes(w.rows, w.cols, dy.rows) : 0;
  if (const Take t = need != 0 ? scratch_workspace(need, a[1], a[5], s, &ws) : given_workspace(a[4], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  // what a small layer can use: scratch of the call, as the partial sums above.  (A given workspace is left alone that is not required.)
  const size_t scratch_bytes = need == 0 && a[4] == Py_None && lib.backward_input_scratch_pays(w.rows, w.cols, dy.rows, y.code, s)
                                   ? lib.backward_input_scratch_bytes(w.rows, w.cols, dy.rows) : 0;
  const uint16_t *wp = pointer<uint16_t>(W), *dyp = pointer<uint16_t>(dY);
  const at::Device device = dY->device();
  const int32_t st = unlocked([&] {
    y.make(device);
    if (scratch_bytes != 0) {
      const Scratch scratch(s, device, scratch_bytes);
      return lib.backward_input_scratch(wp, w.rows, w.cols, w.ld, dyp, dy.rows, dy.ld, y.ptr, y.ld, y.code, scratch.ptr, scratch_bytes, s);
    }
    return lib.backward_input(wp, w.rows, w.cols, w.ld, dyp, dy.rows, dy.ld, y.ptr, y.ld, y.code, ws.ptr, ws.bytes, s);
  });
  return result(st, y.take());
  END_HANDLE_TH_ERRORS
}

// backward_weight(dY, X, mask, out_dtype, out, workspace, stream)
PyObject* backward_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *dY, *X, *mask = nullptr;
  Matrix dy, x;
  Output y;
  void* s;
  if (n != 7 || lib.backward_weight == nullptr || lib.backward_weight_scratch == nullptr ||
      lib.backward_weight_scratch_bytes == nullptr || observed() || !plain(a[0], at::kBFloat16, &dY) ||
      !matrix(*dY, &dy) || !plain(a[1], at::kBFloat16, &X) || !matrix(*X, &x) || x.rows != dy.rows)
    return declined();
  if (a[2] != Py_None && (!plain(a[2], at::kInt, &mask) || !whole(*mask) || mask->size(0) != dy.cols || mask->size(1) != (x.cols + 31) / 32))
    return declined();
  if (!y.read(a[3], a[4], dy.cols, x.cols, false) || !stream_of(a[6], &s)) return declined();
  Workspace ws;
  const size_t need = a[5] == Py_None ? lib.backward_weight_scratch_bytes(dy.cols, x.cols, dy.rows) : 0;
  const auto call = a[5] == Py_None ? lib.backward_weight_scratch : lib.backward_weight;
  if (const Take t = need != 0 ? scratch_workspace(need, a[0], a[6], s, &ws) : given_workspace(a[5], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  const uint16_t *dyp = pointer<uint16_t>(dY), *xp = pointer<uint16_t>(X);
  const uint32_t* mp = pointer<uint32_t>(mask);
  const at::Device device = dY->device();
  const int32_t st = unlocked([&] {
    y.make(device);
    return call(dyp, dy.rows, dy.cols, dy.ld, xp, x.cols, x.ld, mp, y.ptr, y.ld, y.code, ws.ptr, ws.bytes, s);
  });
  return result(st, y.take());
  END_HANDLE_TH_ERRORS
}

bool per_feature(PyObject* obj, int64_t O, const float** out) {
  const at::Tensor* t = nullptr;
  if (obj != Py_None && (!plain(obj, at::kFloat, &t) || t->numel() != O || !t->is_contiguous())) return false;
  *out = pointer<float>(t);
  return true;
}

// forward_i8(Wq, mask, None, N, M, Xq, x_scale, w_scale, bias, out_dtype, out, workspace, stream, prepared), or values, indices and K
// in the first three places
PyObject* forward_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *W, *words, *X;
  Matrix w, x;
  int64_t K, prepared;
  int32_t N, M;
  Output y;
  const float *scale, *bias;
  void* s;
  if (n != 14 || lib.i8_bytes == nullptr || observed() || !plain(a[0], at::kChar, &W) || !plain(a[1], at::kInt, &words) ||
      !whole(*words) || !matrix(*W, &w) || !level(a[3], a[4], &N, &M) || !plain(a[5], at::kChar, &X) || !matrix(*X, &x) ||
      !integer(a[13], 0, 1, &prepared))
    return declined();
  const bool packed = a[2] != Py_None;
  if (packed ? !W->is_contiguous() || !integer(a[2], 1, 1ll << 40, &K)
             : words->size(0) != w.rows || words->size(1) != ((K = w.cols) + 31) / 32)
    return declined();
  const int64_t O = w.rows, T = x.rows;
  if (x.cols != K || !per_feature(a[7], O, &scale) || !per_feature(a[8], O, &bias) || !y.read(a[9], a[10], T, O, true)) return declined();
  float x_scale;
  if (PyFloat_CheckExact(a[6])) x_scale = (float)PyFloat_AS_DOUBLE(a[6]);
  else return declined();
  if (!stream_of(a[12], &s)) return declined();
  Workspace ws;
  const size_t need = a[11] == Py_None ? lib.i8_bytes(O, K, N, M, T) : 0;
  if (need != 0 && prepared) return declined();  // (refused)
  if (const Take t = need != 0 ? scratch_workspace(need, a[5], a[12], s, &ws) : given_workspace(a[11], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  const auto dense_call = prepared ? lib.i8_prepared : lib.i8;
  const auto packed_call = prepared ? lib.i8_packed_prepared : lib.i8_packed;
  if (packed ? packed_call == nullptr : dense_call == nullptr) return declined();
  const int8_t *wp = pointer<int8_t>(W), *xp = pointer<int8_t>(X);
  const uint32_t* mp = pointer<uint32_t>(words);
  const at::Device device = X->device();
  const int32_t st = unlocked([&] {
    y.make(device);
    if (packed) return packed_call(wp, mp, O, K, N, M, xp, T, x.ld, x_scale, scale, bias, y.ptr, y.ld, y.code, ws.ptr, ws.bytes, s);
    return dense_call(wp, O, K, w.ld, mp, N, M, xp, T, x.ld, x_scale, scale, bias, y.ptr, y.ld, y.code, ws.ptr, ws.bytes, s);
  });
  return result(st, y.take());
  END_HANDLE_TH_ERRORS
}

// A float or bfloat16 tensor, and its type code.
bool floating(PyObject* obj, const at::Tensor** t, int32_t* code) {
  if (plain(obj, at::kBFloat16, t)) *code = NM_OUT_BF16;
  else if (plain(obj, at::kFloat, t)) *code = NM_OUT_F32;
  else return false;
  return true;
}
// An optional [rows, cols] matrix of a type.
bool optional_matrix(PyObject* obj, at::ScalarType type, int64_t rows, int64_t cols, const at::Tensor** t, int64_t* ld) {
  *t = nullptr;
  *ld = cols;
  if (obj == Py_None) return true;
  Matrix m;
  if (!plain(obj, type, t) || !matrix(**t, &m) || m.rows != rows || m.cols != cols) return false;
  *ld = m.ld;
  return true;
}
bool flag(PyObject* obj, bool* out) {
  *out = obj == Py_True;
  return PyBool_Check(obj);
}
at::Tensor fresh_like(at::Device device, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
}

// layer_norm(X, weight, bias, eps, residual, train, out_dtype, out, sum_out, stream)
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *X, *R, *S;
  Matrix x;
  int32_t code;
  const float *w, *b;
  int64_t ldr, lds;
  bool train;
  Output y;
  void* s;
  if (n != 10 || lib.layer_norm == nullptr || observed() || !floating(a[0], &X, &code) || !matrix(*X, &x) || !per_feature(a[1], x.cols, &w) ||
      !per_feature(a[2], x.cols, &b) || !PyFloat_CheckExact(a[3]) || !flag(a[5], &train) ||
      !optional_matrix(a[4], X->scalar_type(), x.rows, x.cols, &R, &ldr) ||
      !optional_matrix(a[8], X->scalar_type(), x.rows, x.cols, &S, &lds) || (S != nullptr && R == nullptr) ||
      !y.read(a[6], a[7], x.rows, x.cols, false) || !stream_of(a[9], &s))
    return declined();
  const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
  const at::Device device = X->device();
  const at::ScalarType type = X->scalar_type();
  const void *xp = pointer<void>(X), *rp = pointer<void>(R);
  void* sp = pointer<void>(S);
  at::Tensor sum, stats;
  const int32_t st = unlocked([&] {
    y.make(device);
    if (rp != nullptr && sp == nullptr) {
      sum = fresh(device, x.rows, x.cols, type);
      sp = sum.data_ptr();
    }
    if (train) stats = fresh(device, x.rows, 2, at::kFloat);
    return lib.layer_norm(xp, x.ld, code, rp, ldr, x.rows, x.cols, w, b, eps, y.ptr, y.ld, y.code, sp, lds,
                          train ? static_cast<float*>(stats.data_ptr()) : nullptr, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* out = y.take();
  if (rp == nullptr && !train) return out;
  PyObject* total = nullptr;
  if (rp != nullptr) {
    if (a[8] != Py_None) {
      Py_INCREF(a[8]);
      total = a[8];
    } else {
      total = THPVariable_Wrap(std::move(sum));
    }
  }
  if (!train) return Py_BuildValue("(NN)", out, total);
  PyObject* kept = THPVariable_Wrap(std::move(stats));
  return rp != nullptr ? Py_BuildValue("(NNN)", out, total, kept) : Py_BuildValue("(NN)", out, kept);
  END_HANDLE_TH_ERRORS
}

// layer_norm_backward(dY, S, stats, weight, dS, out_dtype, out, params, workspace, stream)
PyObject* layer_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *dY, *S, *stats, *dS;
  Matrix dy, x;
  int32_t y_code, s_code;
  const float* w;
  int64_t ldds;
  bool params;
  Output d;
  void* s;
  if (n != 10 || lib.layer_norm_backward == nullptr || lib.layer_norm_backward_bytes == nullptr || observed() ||
      !floating(a[0], &dY, &y_code) || !matrix(*dY, &dy) || !floating(a[1], &S, &s_code) || !matrix(*S, &x) || x.rows != dy.rows ||
      x.cols != dy.cols || !plain(a[2], at::kFloat, &stats) || !whole(*stats) || stats->size(0) != dy.rows || stats->size(1) != 2 ||
      !per_feature(a[3], dy.cols, &w) || !optional_matrix(a[4], dY->scalar_type(), dy.rows, dy.cols, &dS, &ldds) ||
      !d.read(a[5], a[6], dy.rows, dy.cols, false) || !flag(a[7], &params) || !stream_of(a[9], &s))
    return declined();
  Workspace ws;
  const size_t need = params && a[8] == Py_None ? lib.layer_norm_backward_bytes(dy.rows, dy.cols) : 0;
  if (const Take t = need != 0 ? scratch_workspace(need, a[0], a[9], s, &ws) : given_workspace(a[8], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  const at::Device device = dY->device();
  const void *dyp = pointer<void>(dY), *xp = pointer<void>(S), *dsp = pointer<void>(dS);
  const float* sp = pointer<float>(stats);
  at::Tensor dw, db;
  const int32_t st = unlocked([&] {
    d.make(device);
    if (params) {
      dw = fresh_like(device, {dy.cols}, at::kFloat);
      db = fresh_like(device, {dy.cols}, at::kFloat);
    }
    return lib.layer_norm_backward(dyp, dy.ld, y_code, xp, x.ld, s_code, sp, w, dsp, ldds, dy.rows, dy.cols, d.ptr, d.ld, d.code,
                                   params ? static_cast<float*>(dw.data_ptr()) : nullptr,
                                   params ? static_cast<float*>(db.data_ptr()) : nullptr, ws.ptr, ws.bytes, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* dx = d.take();
  if (!params) return Py_BuildValue("(NOO)", dx, Py_None, Py_None);
  PyObject* dwp = THPVariable_Wrap(std::move(dw));
  PyObject* dbp = THPVariable_Wrap(std::move(db));
  return Py_BuildValue("(NNN)", dx, dwp, dbp);
  END_HANDLE_TH_ERRORS
}

// [tokens, heads, elements] whose heads are contiguous
bool heads_of(const at::Tensor& t) { return t.dim() == 3 && (t.stride(2) == 1 || t.size(2) <= 1); }

// rotary(X, positions, freqs, sections, interleaved, inverse, out_dtype, out, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor *X, *positions, *freqs, *out = nullptr;
  int32_t code, y_code, sections[4], axes = 1;
  bool interleaved, inverse, whole_numbers;
  void* s;
  if (n != 9 || lib.rotary == nullptr || observed() || !floating(a[0], &X, &code) || !heads_of(*X) ||
      !((whole_numbers = plain(a[1], at::kInt, &positions)) || plain(a[1], at::kFloat, &positions)) || !positions->is_contiguous() ||
      !plain(a[2], at::kFloat, &freqs) || freqs->dim() != 1 || !freqs->is_contiguous() || !flag(a[4], &interleaved) || !flag(a[5], &inverse) ||
      !stream_of(a[8], &s))
    return declined();
  const int64_t T = X->size(0), H = X->size(1), D = X->size(2), pairs = freqs->size(0);
  if (a[3] != Py_None) {
    if (!PyTuple_CheckExact(a[3]) || PyTuple_GET_SIZE(a[3]) < 1 || PyTuple_GET_SIZE(a[3]) > 4) return declined();
    axes = (int32_t)PyTuple_GET_SIZE(a[3]);
    for (int32_t i = 0; i < axes; ++i) {
      int64_t v;
      if (!integer(PyTuple_GET_ITEM(a[3], i), 0, 1 << 30, &v)) return declined();
      sections[i] = (int32_t)v;
    }
  } else {
    if (pairs > 1 << 30) return declined();
    sections[0] = (int32_t)pairs;
  }
  if (positions->dim() == 2 ? positions->size(0) != T || positions->size(1) != axes
                            : positions->dim() != 1 || axes != 1 || positions->size(0) != T)
    return declined();
  at::ScalarType type = X->scalar_type();
  at::Tensor made;
  if (a[7] != Py_None) {
    if (!floating(a[7], &out, &y_code) || !heads_of(*out) || out->size(0) != T || out->size(1) != H || out->size(2) != D) return declined();
  } else {
    if (a[6] != Py_None) {
      if (!THPDtype_Check(a[6])) return declined();
      type = reinterpret_cast<THPDtype*>(a[6])->scalar_type;
    }
    if (type != at::kFloat && type != at::kBFloat16) return declined();
    y_code = type == at::kFloat ? NM_OUT_F32 : NM_OUT_BF16;
  }
  const at::Device device = X->device();
  const int64_t x_token = X->stride(0), x_head = X->stride(1);
  int64_t y_token = out ? out->stride(0) : H * D, y_head = out ? out->stride(1) : D;
  const void *xp = pointer<void>(X), *pp = pointer<void>(positions);
  const float* fp = pointer<float>(freqs);
  void* yp = pointer<void>(out);
  const int32_t st = unlocked([&] {
    if (yp == nullptr) {
      made = fresh_like(device, {T, H, D}, type);
      yp = made.data_ptr();
    }
    return lib.rotary(xp, code, T, H, D, x_token, x_head, pp, !whole_numbers, fp, sections, axes, 2 * pairs, interleaved, inverse, yp,
                      y_code, y_token, y_head, s);
  });
  if (out != nullptr) {
    Py_INCREF(a[7]);
    return result(st, a[7]);
  }
  return result(st, THPVariable_Wrap(std::move(made)));
  END_HANDLE_TH_ERRORS
}

bool read_heads(PyObject* obj, nm_heads* h, const at::Tensor** t) {
  if (!plain(obj, at::kBFloat16, t) || !heads_of(**t)) return false;
  *h = nm_heads{pointer<uint16_t>(*t), (*t)->stride(0), (*t)->stride(1)};
  return true;
}
bool same_sizes(const at::Tensor& a, const at::Tensor& b) { return a.sizes() == b.sizes(); }
// offsets and lengths: an optional int32 [count]
bool per_sequence(PyObject* obj, int64_t count, const int32_t** out) {
  const at::Tensor* t = nullptr;
  if (obj != Py_None && (!plain(obj, at::kInt, &t) || t->dim() != 1 || t->size(0) != count || !t->is_contiguous())) return false;
  *out = pointer<int32_t>(t);
  return true;
}
bool most(PyObject* obj, int64_t otherwise, int64_t* out) {
  *out = otherwise;
  return obj == Py_None || integer(obj, 0, 1ll << 40, out);
}
// what both attention calls have in common: Q, K, V, causal, scale, offsets_q, offsets_k, lengths_k, max_q, max_k from a on
bool read_attention(PyObject* const* a, nm_attention_desc* d, const at::Tensor** Q, const at::Tensor** K) {
  const at::Tensor* V;
  bool causal;
  if (!read_heads(a[0], &d->Q, Q) || !read_heads(a[1], &d->K, K) || !read_heads(a[2], &d->V, &V) || !same_sizes(**K, *V) ||
      (*Q)->size(2) != (*K)->size(2) || !flag(a[3], &causal))
    return false;
  if (a[4] == Py_None) d->scale = (float)(1.0 / std::sqrt((double)(*Q)->size(2)));
  else if (PyFloat_CheckExact(a[4])) d->scale = (float)PyFloat_AS_DOUBLE(a[4]);
  else return false;
  const at::Tensor* first = nullptr;
  int64_t sequences = 1;
  if (a[5] != Py_None) {
    if (a[6] == Py_None || !plain(a[5], at::kInt, &first) || first->dim() != 1 || first->size(0) < 2 || first->size(0) > 1 << 30) return false;
    sequences = first->size(0) - 1;
  } else if (a[6] != Py_None) {
    return false;
  }
  if (!per_sequence(a[5], sequences + 1, &d->offsets_q) || !per_sequence(a[6], sequences + 1, &d->offsets_k) ||
      !per_sequence(a[7], sequences, &d->lengths_k))
    return false;
  d->Tq = (*Q)->size(0);
  d->Tk = (*K)->size(0);
  if (!most(a[8], (d->Tq + sequences - 1) / sequences, &d->max_q) || !most(a[9], (d->Tk + sequences - 1) / sequences, &d->max_k)) return false;
  constexpr int64_t limit = 1 << 30;
  if ((*Q)->size(1) > limit || (*K)->size(1) > limit || (*Q)->size(2) > limit) return false;
  d->sequences = (int32_t)sequences;
  d->heads_q = (int32_t)(*Q)->size(1);
  d->heads_kv = (int32_t)(*K)->size(1);
  d->head_size = (int32_t)(*Q)->size(2);
  d->causal = causal;
  return true;
}
nm_heads contiguous_heads(const at::Tensor& t) {
  return nm_heads{static_cast<uint16_t*>(t.data_ptr()), t.size(1) * t.size(2), t.size(2)};
}

// attention(Q, K, V, causal, scale, offsets_q, offsets_k, lengths_k, max_q, max_k, lse, out, workspace, stream)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_attention_desc d = {};
  const at::Tensor *Q, *K, *O = nullptr;
  bool lse;
  void* s;
  if (n != 14 || lib.attention == nullptr || lib.attention_bytes == nullptr || observed() || !read_attention(a, &d, &Q, &K) ||
      !flag(a[10], &lse) || (a[11] != Py_None && (!read_heads(a[11], &d.O, &O) || !same_sizes(*O, *Q))) || !stream_of(a[13], &s))
    return declined();
  Workspace ws;
  const size_t need = a[12] == Py_None ? lib.attention_bytes(d.Tq, d.sequences, d.heads_q, d.heads_kv, d.head_size, d.max_q,
                                                             d.max_k < d.Tk ? d.max_k : d.Tk) : 0;
  if (const Take t = need != 0 ? scratch_workspace(need, a[0], a[13], s, &ws) : given_workspace(a[12], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  const at::Device device = Q->device();
  const std::vector<int64_t> sizes = Q->sizes().vec();
  at::Tensor made, sums;
  const int32_t st = unlocked([&] {
    if (O == nullptr) {
      made = fresh_like(device, sizes, at::kBFloat16);
      d.O = contiguous_heads(made);
    }
    if (lse) {
      sums = fresh(device, d.heads_q, d.Tq, at::kFloat);
      d.lse = static_cast<float*>(sums.data_ptr());
    }
    return lib.attention(&d, ws.ptr, ws.bytes, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* out;
  if (O != nullptr) {
    Py_INCREF(a[11]);
    out = a[11];
  } else {
    out = THPVariable_Wrap(std::move(made));
  }
  return lse ? Py_BuildValue("(NN)", out, THPVariable_Wrap(std::move(sums))) : out;
  END_HANDLE_TH_ERRORS
}

// attention_backward(dO, Q, K, V, O, lse, causal, scale, offsets_q, offsets_k, lengths_k, max_q, max_k, workspace, stream)
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_attention_desc d = {};
  const at::Tensor *dO, *Q, *K, *O, *lse;
  void* s;
  if (n != 15) return declined();
  PyObject* const shared[10] = {a[1], a[2], a[3], a[6], a[7], a[8], a[9], a[10], a[11], a[12]};
  if (lib.attention_backward == nullptr || lib.attention_backward_bytes == nullptr || observed() || !read_attention(shared, &d, &Q, &K) ||
      !read_heads(a[0], &d.dO, &dO) || !same_sizes(*dO, *Q) || !read_heads(a[4], &d.O, &O) || !same_sizes(*O, *Q) ||
      !plain(a[5], at::kFloat, &lse) || !whole(*lse) || lse->size(0) != d.heads_q || lse->size(1) != d.Tq || !stream_of(a[14], &s))
    return declined();
  d.lse = pointer<float>(lse);
  Workspace ws;
  const size_t need = a[13] == Py_None ? lib.attention_backward_bytes(d.Tq, d.Tk, d.sequences, d.heads_q, d.heads_kv, d.head_size, d.max_q,
                                                                     d.max_k, d.causal) : 0;
  if (const Take t = need != 0 ? scratch_workspace(need, a[1], a[14], s, &ws) : given_workspace(a[13], &ws); t != TAKEN)
    return t == DECLINED ? declined() : nullptr;
  const at::Device device = Q->device();
  const std::vector<int64_t> q_sizes = Q->sizes().vec(), k_sizes = K->sizes().vec();
  at::Tensor dQ, dK, dV;
  const int32_t st = unlocked([&] {
    dQ = fresh_like(device, q_sizes, at::kBFloat16);
    dK = fresh_like(device, k_sizes, at::kBFloat16);
    dV = fresh_like(device, k_sizes, at::kBFloat16);
    d.dQ = contiguous_heads(dQ);
    d.dK = contiguous_heads(dK);
    d.dV = contiguous_heads(dV);
    return lib.attention_backward(&d, ws.ptr, ws.bytes, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* q = THPVariable_Wrap(std::move(dQ));
  PyObject* k = THPVariable_Wrap(std::move(dK));
  PyObject* v = THPVariable_Wrap(std::move(dV));
  return Py_BuildValue("(NNN)", q, k, v);
  END_HANDLE_TH_ERRORS
}

// A head norm's X, weight, heads, eps, centred, positions, freqs, sections, interleaved from a on; `sections` holds what d points to.
bool read_head_norm(PyObject* const* a, nm_head_norm_desc* d, int32_t (&sections)[4], const at::Tensor** X, const at::Tensor** weight) {
  bool centred, interleaved, whole_numbers = false;
  *weight = nullptr;
  if (!floating(a[0], X, &d->X.dtype) || !heads_of(**X) || !PyFloat_CheckExact(a[3]) || !flag(a[4], &centred) || !flag(a[8], &interleaved)) return false;
  d->T = (*X)->size(0);
  d->H = d->heads = (*X)->size(1);
  d->D = (*X)->size(2);
  d->X.data = pointer<void>(*X);
  d->X.token = (*X)->stride(0);
  d->X.head = (*X)->stride(1);
  if (a[2] != Py_None && !integer(a[2], 1, d->H, &d->heads)) return false;
  if (a[1] != Py_None) {
    if (!plain(a[1], at::kFloat, weight) || !(*weight)->is_contiguous()) return false;
    if (d->heads < d->H ? (*weight)->dim() != 2 || (*weight)->size(0) != 2 || (*weight)->size(1) != d->D
                        : (*weight)->dim() != 1 || (*weight)->size(0) != d->D)
      return false;
    d->weight = pointer<float>(*weight);
  }
  d->eps = (float)PyFloat_AS_DOUBLE(a[3]);
  d->centred = centred;
  d->interleaved = interleaved;
  if (a[5] == Py_None) return a[6] == Py_None && a[7] == Py_None;
  const at::Tensor *positions, *freqs;
  if (!((whole_numbers = plain(a[5], at::kInt, &positions)) || plain(a[5], at::kFloat, &positions)) || !positions->is_contiguous() ||
      !plain(a[6], at::kFloat, &freqs) || freqs->dim() != 1 || !freqs->is_contiguous() || freqs->size(0) > 1 << 20)
    return false;
  d->axes = 1;
  sections[0] = (int32_t)freqs->size(0);
  if (a[7] != Py_None) {
    if (!PyTuple_CheckExact(a[7]) || PyTuple_GET_SIZE(a[7]) < 1 || PyTuple_GET_SIZE(a[7]) > 4) return false;
    d->axes = (int32_t)PyTuple_GET_SIZE(a[7]);
    for (int32_t i = 0; i < d->axes; ++i) {
      int64_t v;
      if (!integer(PyTuple_GET_ITEM(a[7], i), 0, 1 << 30, &v)) return false;
      sections[i] = (int32_t)v;
    }
  }
  if (positions->dim() == 2 ? positions->size(0) != d->T || positions->size(1) != d->axes
                            : positions->dim() != 1 || d->axes != 1 || positions->size(0) != d->T)
    return false;
  d->positions = pointer<void>(positions);
  d->positions_f32 = !whole_numbers;
  d->freqs = pointer<float>(freqs);
  d->rotated = 2 * freqs->size(0);
  d->sections = sections;
  return true;
}
// The output of a head norm, or of its backward pass: `out`, or one to be made in X's type or `dtype`.
bool head_norm_output(PyObject* dtype, PyObject* out, const at::Tensor& X, nm_typed_heads* y, at::ScalarType* type) {
  const at::Tensor* t = nullptr;
  *type = X.scalar_type();
  if (out != Py_None) {
    if (!floating(out, &t, &y->dtype) || !heads_of(*t) || t->sizes() != X.sizes()) return false;
    y->data = pointer<void>(t);
    y->token = t->stride(0);
    y->head = t->stride(1);
    return true;
  }
  if (dtype != Py_None) {
    if (!THPDtype_Check(dtype)) return false;
    *type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
  }
  if (*type != at::kFloat && *type != at::kBFloat16) return false;
  y->dtype = *type == at::kFloat ? NM_OUT_F32 : NM_OUT_BF16;
  y->token = X.size(1) * X.size(2);
  y->head = X.size(2);
  return true;
}

// head_norm(X, weight, heads, eps, centred, positions, freqs, sections, interleaved, out_dtype, out, stream)
PyObject* head_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_head_norm_desc d = {};
  int32_t sections[4];
  const at::Tensor *X, *weight;
  at::ScalarType type;
  void* s;
  if (n != 12 || lib.head_norm == nullptr || observed() || !read_head_norm(a, &d, sections, &X, &weight) ||
      !head_norm_output(a[9], a[10], *X, &d.Y, &type) || !stream_of(a[11], &s))
    return declined();
  const at::Device device = X->device();
  at::Tensor made;
  const int32_t st = unlocked([&] {
    if (d.Y.data == nullptr) {
      made = fresh_like(device, {d.T, d.H, d.D}, type);
      d.Y.data = made.data_ptr();
    }
    return lib.head_norm(&d, s);
  });
  if (a[10] != Py_None) {
    Py_INCREF(a[10]);
    return result(st, a[10]);
  }
  return result(st, THPVariable_Wrap(std::move(made)));
  END_HANDLE_TH_ERRORS
}

// head_norm_backward(dY, X, weight, heads, eps, centred, positions, freqs, sections, interleaved, out_dtype, out, params, workspace, stream)
PyObject* head_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_head_norm_desc d = {};
  int32_t sections[4];
  const at::Tensor *X, *weight, *dY;
  at::ScalarType type;
  bool params;
  void* s;
  if (n != 15 || lib.head_norm_backward == nullptr || lib.head_norm_backward_bytes == nullptr || observed() ||
      !read_head_norm(a + 1, &d, sections, &X, &weight) || !floating(a[0], &dY, &d.dY.dtype) || !heads_of(*dY) || dY->sizes() != X->sizes() ||
      !head_norm_output(a[10], a[11], *X, &d.Y, &type) || !flag(a[12], &params) || !stream_of(a[14], &s))
    return declined();
  d.dY.data = pointer<void>(dY);
  d.dY.token = dY->stride(0);
  d.dY.head = dY->stride(1);
  params = params && weight != nullptr;
  Workspace ws;
  if (const Take t = given_workspace(a[13], &ws); t != TAKEN) return t == DECLINED ? declined() : nullptr;
  const size_t need = params && a[13] == Py_None ? lib.head_norm_backward_bytes(d.T, d.H, d.heads, d.D, d.rotated) : 0;
  const at::Device device = X->device();
  const std::vector<int64_t> sizes = params ? weight->sizes().vec() : std::vector<int64_t>();
  at::Tensor made, dw;
  const int32_t st = unlocked([&] {
    if (d.Y.data == nullptr) {
      made = fresh_like(device, {d.T, d.H, d.D}, type);
      d.Y.data = made.data_ptr();
    }
    if (params) {
      dw = fresh_like(device, sizes, at::kFloat);
      d.dweight = static_cast<float*>(dw.data_ptr());
    }
    if (need == 0) return lib.head_norm_backward(&d, ws.ptr, ws.bytes, s);
    const Scratch own(s, device, need);
    return lib.head_norm_backward(&d, own.ptr, need, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* dx;
  if (a[11] != Py_None) {
    Py_INCREF(a[11]);
    dx = a[11];
  } else {
    dx = THPVariable_Wrap(std::move(made));
  }
  if (!params) return Py_BuildValue("(NO)", dx, Py_None);
  PyObject* dwp = THPVariable_Wrap(std::move(dw));
  return Py_BuildValue("(NN)", dx, dwp);
  END_HANDLE_TH_ERRORS
}

// A cache in pages: K_pages, V_pages, page_table, lengths; K_scales, V_scales.
bool read_pages(PyObject* const* a, PyObject* k_scales, PyObject* v_scales, nm_pages* p, const at::Tensor** K) {
  const at::Tensor *V, *table, *ks, *vs;
  if (plain(a[0], at::kFloat8_e4m3fn, K)) p->dtype = NM_E4M3;
  else if (plain(a[0], at::kBFloat16, K)) p->dtype = NM_OUT_BF16;
  else return false;
  if (!plain(a[1], (*K)->scalar_type(), &V) || (*K)->dim() != 4 || (*K)->sizes() != V->sizes() || (*K)->strides() != V->strides() ||
      ((*K)->stride(3) != 1 && (*K)->size(3) > 1))
    return false;
  constexpr int64_t limit = 1 << 30;
  for (int i = 1; i < 4; ++i)
    if ((*K)->size(i) > limit) return false;
  p->pages = (*K)->size(0);
  p->page_size = (int32_t)(*K)->size(1);
  p->heads = (int32_t)(*K)->size(2);
  p->head_size = (int32_t)(*K)->size(3);
  p->page = (*K)->stride(0);
  p->token = (*K)->stride(1);
  p->head = (*K)->stride(2);
  p->K = pointer<void>(*K);
  p->V = pointer<void>(V);
  if (p->dtype == NM_E4M3) {
    if (!plain(k_scales, at::kByte, &ks) || !plain(v_scales, at::kByte, &vs) || ks->dim() != 3 || ks->sizes() != (*K)->sizes().slice(0, 3) ||
        vs->sizes() != ks->sizes() || vs->strides() != ks->strides())
      return false;
    p->scale_page = ks->stride(0);
    p->scale_token = ks->stride(1);
    p->scale_head = ks->stride(2);
    p->K_scales = pointer<uint8_t>(ks);
    p->V_scales = pointer<uint8_t>(vs);
  } else if (k_scales != Py_None || v_scales != Py_None) {
    return false;
  }
  if (!plain(a[2], at::kInt, &table) || !whole(*table) || table->size(0) > limit || table->size(1) > limit) return false;
  p->sequences = (int32_t)table->size(0);
  p->table_width = (int32_t)table->size(1);
  p->table = pointer<int32_t>(table);
  return per_sequence(a[3], p->sequences, &p->lengths) && p->lengths != nullptr;
}
bool packed_tokens(PyObject* obj, const nm_pages& p, nm_heads* h, int64_t* tokens) {
  const at::Tensor* t;
  if (!read_heads(obj, h, &t) || t->size(1) != p.heads || t->size(2) != p.head_size) return false;
  if (*tokens < 0) *tokens = t->size(0);
  return t->size(0) == *tokens;
}

// cache_write(K, V, K_pages, V_pages, page_table, lengths, offsets, K_scales, V_scales, stream)
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_pages p = {};
  nm_heads K, V;
  const at::Tensor* pages;
  const int32_t* offsets;
  int64_t T = -1;
  void* s;
  if (n != 10 || lib.cache_write == nullptr || observed() || !read_pages(a + 2, a[7], a[8], &p, &pages) || !packed_tokens(a[0], p, &K, &T) ||
      !packed_tokens(a[1], p, &V, &T) || !per_sequence(a[6], p.sequences + 1, &offsets) || !stream_of(a[9], &s))
    return declined();
  const int32_t st = unlocked([&] { return lib.cache_write(&p, &K, &V, offsets, T, s); });
  Py_INCREF(Py_None);
  return result(st, Py_None);
  END_HANDLE_TH_ERRORS
}

// cache_read(K_pages, V_pages, page_table, lengths, offsets, tokens, first, K_scales, V_scales, out, stream)
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_pages p = {};
  nm_heads K = {}, V = {};
  const at::Tensor* pages;
  const int32_t *offsets, *first;
  int64_t T = -1;
  void* s;
  if (n != 11 || lib.cache_read == nullptr || observed() || !read_pages(a, a[7], a[8], &p, &pages) ||
      (a[5] != Py_None && !integer(a[5], 0, 1 << 30, &T)) || !per_sequence(a[4], p.sequences + 1, &offsets) ||
      !per_sequence(a[6], p.sequences, &first) || !stream_of(a[10], &s))
    return declined();
  const bool given = a[9] != Py_None;
  if (given ? !PyTuple_CheckExact(a[9]) || PyTuple_GET_SIZE(a[9]) != 2 || !packed_tokens(PyTuple_GET_ITEM(a[9], 0), p, &K, &T) ||
                  !packed_tokens(PyTuple_GET_ITEM(a[9], 1), p, &V, &T)
            : T < 0)
    return declined();
  const at::Device device = pages->device();
  at::Tensor k, v;
  const int32_t st = unlocked([&] {
    if (!given) {
      k = fresh_like(device, {T, p.heads, p.head_size}, at::kBFloat16);
      v = fresh_like(device, {T, p.heads, p.head_size}, at::kBFloat16);
      K = contiguous_heads(k);
      V = contiguous_heads(v);
    }
    return lib.cache_read(&p, &K, &V, offsets, first, T, s);
  });
  if (given) {
    Py_INCREF(a[9]);
    return result(st, a[9]);
  }
  if (st != NM_OK) return result(st, nullptr);
  PyObject* kp = THPVariable_Wrap(std::move(k));
  PyObject* vp = THPVariable_Wrap(std::move(v));
  return Py_BuildValue("(NN)", kp, vp);
  END_HANDLE_TH_ERRORS
}

// attention_paged(Q, K_pages, V_pages, page_table, lengths, scale, offsets_q, window, sinks, K_scales, V_scales, max_q, max_k, lse, out,
//                 workspace, stream)
PyObject* attention_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  nm_paged_desc d = {};
  const at::Tensor *Q, *pages, *O = nullptr;
  bool lse;
  int64_t window, sinks;
  void* s;
  if (n != 17 || lib.attention_paged == nullptr || lib.attention_paged_bytes == nullptr || observed() || !read_heads(a[0], &d.Q, &Q) ||
      !read_pages(a + 1, a[9], a[10], &d.pages, &pages) || Q->size(2) != d.pages.head_size || Q->size(1) > 1 << 30 ||
      !per_sequence(a[6], d.pages.sequences + 1, &d.offsets_q) || !integer(a[7], 0, 1 << 30, &window) || !integer(a[8], 0, 1 << 30, &sinks) ||
      d.pages.sequences < 1 || !most(a[11], (Q->size(0) + d.pages.sequences - 1) / d.pages.sequences, &d.max_q) ||
      !most(a[12], (int64_t)d.pages.table_width * d.pages.page_size, &d.max_k) || !flag(a[13], &lse) ||
      (a[14] != Py_None && (!read_heads(a[14], &d.O, &O) || !same_sizes(*O, *Q))) || !stream_of(a[16], &s))
    return declined();
  if (a[5] == Py_None) d.scale = (float)(1.0 / std::sqrt((double)Q->size(2)));
  else if (PyFloat_CheckExact(a[5])) d.scale = (float)PyFloat_AS_DOUBLE(a[5]);
  else return declined();
  d.Tq = Q->size(0);
  d.heads_q = (int32_t)Q->size(1);
  d.window = (int32_t)window;
  d.sinks = (int32_t)sinks;
  Workspace ws;
  if (const Take t = given_workspace(a[15], &ws); t != TAKEN) return t == DECLINED ? declined() : nullptr;
  const size_t need = a[15] == Py_None ? lib.attention_paged_bytes(d.Tq, d.pages.sequences, d.heads_q, d.pages.heads, d.pages.head_size, d.max_q) : 0;
  const at::Device device = Q->device();
  const std::vector<int64_t> sizes = Q->sizes().vec();
  at::Tensor made, sums;
  const int32_t st = unlocked([&] {
    if (O == nullptr) {
      made = fresh_like(device, sizes, at::kBFloat16);
      d.O = contiguous_heads(made);
    }
    if (lse) {
      sums = fresh(device, d.heads_q, d.Tq, at::kFloat);
      d.lse = static_cast<float*>(sums.data_ptr());
    }
    if (need == 0) return lib.attention_paged(&d, ws.ptr, ws.bytes, s);
    const Scratch own(s, device, need);
    return lib.attention_paged(&d, own.ptr, need, s);
  });
  if (st != NM_OK) return result(st, nullptr);
  PyObject* out;
  if (O != nullptr) {
    Py_INCREF(a[14]);
    out = a[14];
  } else {
    out = THPVariable_Wrap(std::move(made));
  }
  return lse ? Py_BuildValue("(NN)", out, THPVariable_Wrap(std::move(sums))) : out;
  END_HANDLE_TH_ERRORS
}

// bind(addresses by name, raise_status, find_workspace[, where that keeps its tensors])
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *table, *raise, *find, *kept = nullptr;
  if (!PyArg_ParseTuple(args, "O!OO|O!", &PyDict_Type, &table, &raise, &find, &PyDict_Type, &kept)) return nullptr;
  Library l = {};
  struct { const char* name; void* slot; bool optional = false; } slots[] = {
      {"nm_prune", &l.prune}, {"nm_prune_scored", &l.prune_scored}, {"nm_pack", &l.pack}, {"nm_unpack", &l.unpack},
      {"nm_linear_forward", &l.forward}, {"nm_linear_forward_prepared", &l.forward_prepared},
      {"nm_linear_forward_static", &l.forward_static}, {"nm_spmm_workspace_bytes", &l.workspace_bytes},
      {"nm_values_bytes", &l.values_bytes}, {"nm_index_bytes", &l.index_bytes},
      {"nm_linear_forward_prepared_scratch", &l.forward_prepared_scratch, true},
      {"nm_prepared_scratch_bytes", &l.prepared_scratch_bytes, true},
      {"nm_linear_backward_input", &l.backward_input, true}, {"nm_linear_backward_weight", &l.backward_weight, true},
      {"nm_linear_backward_input_scratch", &l.backward_input_scratch, true},
      {"nm_backward_input_workspace_bytes", &l.backward_input_bytes, true},
      {"nm_backward_input_scratch_bytes", &l.backward_input_scratch_bytes, true},
      {"nm_backward_input_scratch_pays", &l.backward_input_scratch_pays, true},
      {"nm_linear_backward_weight_scratch", &l.backward_weight_scratch, true},
      {"nm_backward_weight_scratch_bytes", &l.backward_weight_scratch_bytes, true}, {"nm_linear_forward_i8", &l.i8, true},
      {"nm_linear_forward_i8_prepared", &l.i8_prepared, true}, {"nm_linear_forward_i8_packed", &l.i8_packed, true},
      {"nm_linear_forward_i8_packed_prepared", &l.i8_packed_prepared, true}, {"nm_i8_workspace_bytes", &l.i8_bytes, true},
      {"nm_layer_norm", &l.layer_norm, true}, {"nm_layer_norm_backward", &l.layer_norm_backward, true},
      {"nm_layer_norm_backward_workspace_bytes", &l.layer_norm_backward_bytes, true}, {"nm_rotary", &l.rotary, true},
      {"nm_attention", &l.attention, true}, {"nm_attention_workspace_bytes", &l.attention_bytes, true},
      {"nm_attention_backward", &l.attention_backward, true},
      {"nm_attention_backward_workspace_bytes", &l.attention_backward_bytes, true},
      {"nm_head_norm", &l.head_norm, true}, {"nm_head_norm_backward", &l.head_norm_backward, true},
      {"nm_head_norm_backward_workspace_bytes", &l.head_norm_backward_bytes, true}, {"nm_cache_write", &l.cache_write, true},
      {"nm_cache_read", &l.cache_read, true}, {"nm_attention_paged", &l.attention_paged, true},
      {"nm_attention_paged_workspace_bytes", &l.attention_paged_bytes, true}};
  for (auto& e : slots) {
    PyObject* address = PyDict_GetItemString(table, e.name);
    if (address == nullptr && e.optional) continue;
    void* p = address ? PyLong_AsVoidPtr(address) : nullptr;
    if (p == nullptr) {
      if (!PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "%s", e.name);
      return nullptr;
    }
    *static_cast<void**>(e.slot) = p;
  }
  lib = l;
  Py_INCREF(raise);
  Py_XSETREF(raise_status, raise);
  Py_INCREF(find);
  Py_XSETREF(find_workspace, find);
  Py_XINCREF(kept);
  Py_XSETREF(workspaces, kept);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"prune", (PyCFunction)(void (*)())prune, METH_FASTCALL, nullptr},
    {"prune_scored", (PyCFunction)(void (*)())prune_scored, METH_FASTCALL, nullptr},
    {"pack", (PyCFunction)(void (*)())pack, METH_FASTCALL, nullptr},
    {"unpack", (PyCFunction)(void (*)())unpack, METH_FASTCALL, nullptr},
    {"forward", (PyCFunction)(void (*)())forward, METH_FASTCALL, nullptr},
    {"backward_input", (PyCFunction)(void (*)())backward_input, METH_FASTCALL, nullptr},
    {"backward_weight", (PyCFunction)(void (*)())backward_weight, METH_FASTCALL, nullptr},
    {"forward_i8", (PyCFunction)(void (*)())forward_i8, METH_FASTCALL, nullptr},
    {"layer_norm", (PyCFunction)(void (*)())layer_norm, METH_FASTCALL, nullptr},
    {"layer_norm_backward", (PyCFunction)(void (*)())layer_norm_backward, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void (*)())rotary, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, nullptr},
    {"attention_backward", (PyCFunction)(void (*)())attention_backward, METH_FASTCALL, nullptr},
    {"head_norm", (PyCFunction)(void (*)())head_norm, METH_FASTCALL, nullptr},
    {"head_norm_backward", (PyCFunction)(void (*)())head_norm_backward, METH_FASTCALL, nullptr},
    {"cache_write", (PyCFunction)(void (*)())cache_write, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void (*)())cache_read, METH_FASTCALL, nullptr},
    {"attention_paged", (PyCFunction)(void (*)())attention_paged, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_nm_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nm_calls() { return PyModule_Create(&module); }
