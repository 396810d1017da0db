// Marshalling of the hot entry points in native code: checks of the tensors, allocation of the results and the call into
// the C ABI, for binding.py.  No arithmetic of the path lives here; the library's functions come in as addresses, so this
// module is tied to whichever libfp4attn.so binding.py has loaded.
//
// Why: a step of the smallest problems is four kernels of 2-8 us each, and the same marshalling in Python (ctypes, size
// queries, torch.empty, stream look-up) took about 15 us per call: B=1, H=2, N=256 ran at 66 us per step, all of it host
// time.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <limits>

#include "../../include/fp4attn.h"

namespace {

struct Api {
  decltype(&fp4attn_status_string) status_string;
  decltype(&fp4attn_packed_bytes) packed_bytes;
  decltype(&fp4attn_scale_bytes) scale_bytes;
  decltype(&fp4attn_quantize_workspace_bytes) quantize_workspace_bytes;
  decltype(&fp4attn_quantize) quantize;
  decltype(&fp4attn_quantize_mxfp4_rule) quantize_mxfp4_rule;
  decltype(&fp4attn_quantize_nvfp4_per_head_workspace_bytes) per_head_workspace_bytes;
  decltype(&fp4attn_quantize_nvfp4_per_head) per_head;
  decltype(&fp4attn_quantize_v_e4m3_workspace_bytes) e4m3_workspace_bytes;
  decltype(&fp4attn_quantize_v_e4m3) e4m3;
  decltype(&fp4attn_fwd) fwd;
  decltype(&fp4attn_rotary) rotary;
  decltype(&fp4attn_cache_record_bytes) cache_record_bytes;
  decltype(&fp4attn_cache_write) cache_write;
  decltype(&fp4attn_cache_read) cache_read;
  decltype(&fp4attn_tree_attention_workspace_bytes) tree_workspace_bytes;
  decltype(&fp4attn_tree_attention) tree_attention;
  decltype(&fp4attn_paged_attention_workspace_bytes) paged_workspace_bytes;
  decltype(&fp4attn_paged_attention) paged_attention;
  decltype(&fp4attn_shared_prefix_attention_workspace_bytes) shared_workspace_bytes;
  decltype(&fp4attn_shared_prefix_attention) shared_prefix_attention;
  decltype(&fp4attn_pages_assign) pages_assign;
  decltype(&fp4attn_pages_release_workspace_bytes) release_workspace_bytes;
  decltype(&fp4attn_pages_release) pages_release;
};
Api g_api;
PyObject* g_error = nullptr;                            // Fp4AttnError
enum { A_PACKED, A_SCALES, A_G, A_FMT, A_ROLE, A_SHAPE, A_PER_HEAD, A_COUNT };
enum { C_PAGES, C_K_G, C_V_G, C_FMT, C_PAGE_SIZE, C_D, C_COUNT };
enum { P_FREE, P_COUNT_OF, P_TURN, P_PAGE_SIZE, P_COUNT };
PyObject* g_cache_names[C_COUNT];
PyObject* g_pool_names[P_COUNT];
PyObject* g_names[A_COUNT];
constexpr int kFmtE4m3 = 2;                             // QuantizedOperand.fmt of an E4M3 V

PyObject* fail(int rc, const char* what) {
  PyErr_Format(g_error, "%s: %s (status %d)", what, g_api.status_string(rc), rc);
  return nullptr;
}
PyObject* assertion(const char* what) {
  PyErr_SetString(PyExc_AssertionError, what);
  return nullptr;
}
fp4attn_stream_t stream() { return reinterpret_cast<fp4attn_stream_t>(c10::cuda::getCurrentCUDAStream().stream()); }
at::Tensor device_empty(at::IntArrayRef size, at::ScalarType type, c10::Device device) {
  return at::Tensor(at::detail::empty_cuda(size, type, device, std::nullopt));
}
// The results of one call.  An allocation costs about as much host time as the rest of a call's marshalling, so up to
// kShareBytes they are pieces of one (a step of B=1, H=2, N=256: 19.9 -> 17.0 us); beyond that (where the kernels take longer anyway) each has memory of its own, so that
// keeping one alone does not keep them all.
struct Results {
  static constexpr size_t kShareBytes = 1 << 20, kMost = 4;
  struct Piece {
    int64_t sizes[4];
    int dims;
    at::ScalarType type;
    at::Tensor tensor;
  } piece[kMost];
  int n = 0;
  at::Tensor& add(std::initializer_list<int64_t> sizes, at::ScalarType type) {
    Piece& p = piece[n++];
    p.dims = (int)sizes.size();
    p.type = type;
    std::copy(sizes.begin(), sizes.end(), p.sizes);
    return p.tensor;
  }
  void allocate(c10::Device device) {
    int64_t at[kMost + 1] = {0}, count[kMost];
    for (int i = 0; i < n; ++i) {
      count[i] = 1;
      for (int k = 0; k < piece[i].dims; ++k) count[i] *= piece[i].sizes[k];
      at[i + 1] = at[i] + ((count[i] * (int64_t)c10::elementSize(piece[i].type) + 511) & ~511ll);   // as the allocator aligns
    }
    if (at[n] > (int64_t)kShareBytes) {
      for (int i = 0; i < n; ++i) piece[i].tensor = device_empty(at::IntArrayRef(piece[i].sizes, piece[i].dims), piece[i].type, device);
      return;
    }
    // straight from the caching allocator: a tensor of its own for the block would only be taken apart again
    const c10::cuda::OptionalCUDAGuard guard(device);
    c10::Allocator* const pool = c10::cuda::CUDACachingAllocator::get();
    const c10::Storage block(c10::Storage::use_byte_size_t(), (size_t)at[n], pool->allocate((size_t)at[n]), pool, /*resizable=*/true);
    for (int i = 0; i < n; ++i) {
      piece[i].tensor = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(block), c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(piece[i].type));
      c10::TensorImpl* impl = piece[i].tensor.unsafeGetTensorImpl();
      impl->set_sizes_contiguous(at::IntArrayRef(piece[i].sizes, piece[i].dims));
      impl->set_storage_offset(at[i] / (int64_t)c10::elementSize(piece[i].type));
    }
  }
};
// What a Python caller's `None if o is None else o.data_ptr()` gives: a null pointer for None, and an error for what has no
// memory (an argument that is not a tensor must not pass for one that was left out).
bool data_of(PyObject* o, void** ptr) {
  *ptr = nullptr;
  if (o == Py_None) return true;
  if (THPVariable_Check(o)) {
    *ptr = THPVariable_Unpack(o).data_ptr();
    return true;
  }
  PyObject* p = PyObject_CallMethod(o, "data_ptr", nullptr);
  if (p) *ptr = PyLong_AsVoidPtr(p);
  Py_XDECREF(p);
  return !PyErr_Occurred();
}
bool numel_of(PyObject* o, size_t* n) {
  if (THPVariable_Check(o)) {
    *n = (size_t)THPVariable_Unpack(o).numel();
    return true;
  }
  PyObject* p = PyObject_CallMethod(o, "numel", nullptr);
  if (p) *n = PyLong_AsSize_t(p);
  Py_XDECREF(p);
  return !PyErr_Occurred();
}

struct Input {
  const at::Tensor* t = nullptr;
  int B = 0, H = 0, N = 0, d = 0;
  bool take(PyObject* o) {
    if (!THPVariable_Check(o)) return false;
    t = &THPVariable_Unpack(o);
    if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || t->dim() != 4 || !t->is_contiguous()) return false;
    const auto s = t->sizes();
    for (int i = 0; i < 4; ++i)
      if (s[i] > INT32_MAX) return false;
    B = (int)s[0]; H = (int)s[1]; N = (int)s[2]; d = (int)s[3];
    return true;
  }
  PyObject* shape() const { return Py_BuildValue("(iiii)", B, H, N, d); }
};
const char* kInputRule = "x must be a contiguous CUDA bfloat16 tensor [B, H, N, d]";

// (packed, scales, G or None, shape)
PyObject* result(const at::Tensor& packed, const at::Tensor* scales, const at::Tensor* G, const Input& in) {
  PyObject* g = G ? THPVariable_Wrap(*G) : Py_NewRef(Py_None);
  PyObject* s = scales ? THPVariable_Wrap(*scales) : Py_NewRef(Py_None);
  return Py_BuildValue("(NNNN)", THPVariable_Wrap(packed), s, g, in.shape());
}

// whole numbers; `convert`: whatever int() takes
bool ints(PyObject* const* args, Py_ssize_t n, int* out, bool convert = false) {
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!convert && !PyLong_Check(args[i])) {
      PyErr_Format(PyExc_TypeError, "int expected instead of %s instance", Py_TYPE(args[i])->tp_name);
      return false;
    }
    PyObject* o = PyLong_Check(args[i]) ? Py_NewRef(args[i]) : PyNumber_Long(args[i]);
    const long v = o ? PyLong_AsLong(o) : -1;
    Py_XDECREF(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT32_MIN || v > INT32_MAX) {                // (cut to 32 bits it would be another number, and pass)
      PyErr_SetString(PyExc_OverflowError, "int does not fit 32 bits");
      return false;
    }
    out[i] = (int)v;
  }
  return true;
}
bool number(PyObject* o, float* out) {                  // whatever float() takes
  PyObject* f = PyNumber_Float(o);
  if (f) *out = (float)PyFloat_AsDouble(f);
  Py_XDECREF(f);
  return f != nullptr;
}
// A call into the library, which may block on a full launch queue, without the interpreter lock (nothing in it may touch a
// Python object).
template <class F>
int unlocked(F call) {
  struct Unlock {
    PyThreadState* ts = PyEval_SaveThread();
    ~Unlock() { PyEval_RestoreThread(ts); }
  } guard;
  return call();
}

#define FP4_TRY try {
#define FP4_CATCH                                                                              \
  }                                                                                            \
  catch (const c10::OutOfMemoryError& e) {                                                     \
    PyErr_SetString(out_of_memory_class(), e.what_without_backtrace());                   \
    return nullptr;                                                                            \
  }                                                                                            \
  catch (const std::exception& e) {                                                            \
    PyErr_SetString(PyExc_RuntimeError, e.what());                                             \
    return nullptr;                                                                            \
  }
PyObject* out_of_memory_class() {                       // torch.OutOfMemoryError
  static PyObject* cls = [] {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* c = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    Py_XDECREF(torch);
    return c ? c : PyExc_RuntimeError;
  }();
  return cls;
}

// quantize(x, fmt, role, workspace)
PyObject* py_quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  int a[2];
  Input in;
  if (n != 4 || !in.take(args[0])) return assertion(kInputRule);
  if (!ints(args + 1, 2, a)) return nullptr;
  const int fmt = a[0], role = a[1];
  const size_t nb = g_api.packed_bytes(in.B, in.H, in.N, in.d), ns = g_api.scale_bytes(fmt, role, in.B, in.H, in.N, in.d);
  void* const any = reinterpret_cast<void*>(1);
  if (!nb || !ns) {                                     // unsupported: the library says why, before it looks at a pointer's use
    const int rc = unlocked([&] { return g_api.quantize(in.t->data_ptr(), fmt, role, in.B, in.H, in.N, in.d, any, any, nullptr, nullptr, 0, stream()); });
    if (rc) return fail(rc, "fp4attn_quantize");
    PyErr_SetString(g_error, "fp4attn_quantize: unsupported arguments");
    return nullptr;
  }
  const size_t nw = args[3] == Py_None ? g_api.quantize_workspace_bytes(fmt, role, in.B, in.H, in.N, in.d) : 0;
  Results r;
  at::Tensor none, &packed = r.add({(int64_t)nb}, at::kByte), &scales = r.add({(int64_t)ns}, at::kByte);
  at::Tensor& G = fmt == FP4ATTN_FMT_NVFP4 ? r.add({1}, at::kFloat) : none;
  at::Tensor& ws = nw ? r.add({(int64_t)nw}, at::kByte) : none;
  void* wptr = nullptr;
  size_t wbytes = nw;
  if (args[3] != Py_None && (!data_of(args[3], &wptr) || !numel_of(args[3], &wbytes))) return nullptr;
  r.allocate(in.t->device());
  if (nw) wptr = ws.data_ptr();
  const int rc = unlocked([&] { return g_api.quantize(in.t->data_ptr(), fmt, role, in.B, in.H, in.N, in.d, packed.data_ptr(), scales.data_ptr(),
                                G.defined() ? G.data_ptr<float>() : nullptr, wptr, wbytes, stream()); });
  if (rc) return fail(rc, "fp4attn_quantize");
  return result(packed, &scales, G.defined() ? &G : nullptr, in);
  FP4_CATCH
}

// quantize_mxfp4_rule(x, role, scale_rule)
PyObject* py_rule(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  int a[2];
  Input in;
  if (n != 3 || !in.take(args[0])) return assertion(kInputRule);
  if (!ints(args + 1, 2, a)) return nullptr;
  const size_t nb = g_api.packed_bytes(in.B, in.H, in.N, in.d), ns = g_api.scale_bytes(FP4ATTN_FMT_MXFP4, a[0], in.B, in.H, in.N, in.d);
  void* const any = reinterpret_cast<void*>(1);
  if (!nb || !ns) {
    const int rc = unlocked([&] { return g_api.quantize_mxfp4_rule(in.t->data_ptr(), a[0], a[1], in.B, in.H, in.N, in.d, any, any, stream()); });
    if (rc) return fail(rc, "fp4attn_quantize_mxfp4_rule");
    PyErr_SetString(g_error, "fp4attn_quantize_mxfp4_rule: unsupported arguments");
    return nullptr;
  }
  Results r;
  at::Tensor &packed = r.add({(int64_t)nb}, at::kByte), &scales = r.add({(int64_t)ns}, at::kByte);
  r.allocate(in.t->device());
  const int rc = unlocked([&] { return g_api.quantize_mxfp4_rule(in.t->data_ptr(), a[0], a[1], in.B, in.H, in.N, in.d, packed.data_ptr(), scales.data_ptr(), stream()); });
  if (rc) return fail(rc, "fp4attn_quantize_mxfp4_rule");
  return result(packed, &scales, nullptr, in);
  FP4_CATCH
}

// quantize_nvfp4_per_head(x, role)
PyObject* py_per_head(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  int role;
  Input in;
  if (n != 2 || !in.take(args[0])) return assertion(kInputRule);
  if (!ints(args + 1, 1, &role)) return nullptr;
  const size_t nb = g_api.packed_bytes(in.B, in.H, in.N, in.d), ns = g_api.scale_bytes(FP4ATTN_FMT_NVFP4, role, in.B, in.H, in.N, in.d);
  const size_t nw = g_api.per_head_workspace_bytes(in.B, in.H, in.N, in.d);
  void* const any = reinterpret_cast<void*>(1);
  if (!nb || !ns || !nw) {
    const int rc = unlocked([&] { return g_api.per_head(in.t->data_ptr(), role, in.B, in.H, in.N, in.d, any, any, reinterpret_cast<float*>(any), nullptr, 0, stream()); });
    if (rc) return fail(rc, "fp4attn_quantize_nvfp4_per_head");
    PyErr_SetString(g_error, "fp4attn_quantize_nvfp4_per_head: unsupported arguments");
    return nullptr;
  }
  Results r;
  at::Tensor &packed = r.add({(int64_t)nb}, at::kByte), &scales = r.add({(int64_t)ns}, at::kByte);
  at::Tensor &G = r.add({(int64_t)in.B * in.H}, at::kFloat), &ws = r.add({(int64_t)nw}, at::kByte);
  r.allocate(in.t->device());
  const int rc = unlocked([&] { return g_api.per_head(in.t->data_ptr(), role, in.B, in.H, in.N, in.d, packed.data_ptr(), scales.data_ptr(), G.data_ptr<float>(),
                                ws.data_ptr(), nw, stream()); });
  if (rc) return fail(rc, "fp4attn_quantize_nvfp4_per_head");
  return result(packed, &scales, &G, in);
  FP4_CATCH
}

// quantize_v_e4m3(x); scales comes back empty
PyObject* py_e4m3(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  Input in;
  if (n != 1 || !in.take(args[0])) return assertion(kInputRule);
  const size_t nw = g_api.e4m3_workspace_bytes(in.B, in.H, in.N, in.d);
  void* const any = reinterpret_cast<void*>(1);
  if (!nw) {
    const int rc = unlocked([&] { return g_api.e4m3(in.t->data_ptr(), in.B, in.H, in.N, in.d, any, reinterpret_cast<float*>(any), nullptr, 0, stream()); });
    if (rc) return fail(rc, "fp4attn_quantize_v_e4m3");
    PyErr_SetString(g_error, "fp4attn_quantize_v_e4m3: unsupported arguments");
    return nullptr;
  }
  Results r;
  at::Tensor &out = r.add({in.t->numel()}, at::kByte), &scales = r.add({0}, at::kByte);
  at::Tensor &G = r.add({(int64_t)in.B * in.H}, at::kFloat), &ws = r.add({(int64_t)nw}, at::kByte);
  r.allocate(in.t->device());
  const int rc = unlocked([&] { return g_api.e4m3(in.t->data_ptr(), in.B, in.H, in.N, in.d, out.data_ptr(), G.data_ptr<float>(), ws.data_ptr(), nw, stream()); });
  if (rc) return fail(rc, "fp4attn_quantize_v_e4m3");
  return result(out, &scales, &G, in);
  FP4_CATCH
}

// What fp4attn_fwd reads of a QuantizedOperand.  The tensors stay alive through the operand, which the caller holds.
struct Operand {
  void *packed = nullptr, *scales = nullptr, *G = nullptr;
  c10::Device device{c10::kCPU};
  int fmt = 0, shape[4] = {0, 0, 0, 0};
  bool per_head = false;
  bool take(PyObject* o) {
    PyObject* v[A_COUNT] = {};
    bool ok = true;
    for (int i = 0; i < A_COUNT && ok; ++i) {
      if (i == A_ROLE) continue;
      v[i] = PyObject_GetAttr(o, g_names[i]);
      ok = v[i] != nullptr;
    }
    if (ok && !PyTuple_Check(v[A_SHAPE])) {
      PyObject* const t = PySequence_Tuple(v[A_SHAPE]);
      Py_SETREF(v[A_SHAPE], t);
      ok = t != nullptr;
    }
    if (ok && (!THPVariable_Check(v[A_PACKED]) || PyTuple_GET_SIZE(v[A_SHAPE]) != 4)) {
      PyErr_SetString(PyExc_TypeError, "fp4attn_fwd takes QuantizedOperand arguments");
      ok = false;
    }
    if (ok) {
      const at::Tensor& t = THPVariable_Unpack(v[A_PACKED]);
      packed = t.data_ptr();
      device = t.device();
      if (!data_of(v[A_SCALES], &scales) || !data_of(v[A_G], &G)) ok = false;
      fmt = ok ? (int)PyLong_AsLong(v[A_FMT]) : 0;
      per_head = ok && PyObject_IsTrue(v[A_PER_HEAD]) == 1;
      for (int i = 0; ok && i < 4; ++i) shape[i] = (int)PyLong_AsLong(PyTuple_GET_ITEM(v[A_SHAPE], i));
      ok = ok && !PyErr_Occurred();
    }
    for (int i = 0; i < A_COUNT; ++i) Py_XDECREF(v[i]);
    return ok;
  }
};

// fwd(q, k, v, softmax_scale, out, lse, status, p_map, affine_a, affine_b, p_scale_rule, causal, exact_pairs, schedule, seq_len,
//     fixed_reference) -> (out, lse)
PyObject* py_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 16) return assertion("fwd takes 16 arguments");
  Operand q, k, v;
  if (!q.take(args[0]) || !k.take(args[1]) || !v.take(args[2])) return nullptr;
  const int B = q.shape[0], H = q.shape[1], N = q.shape[2], d = q.shape[3], Hkv = k.shape[1];
  bool same = k.shape[0] == B && k.shape[2] == N && k.shape[3] == d && Hkv > 0 && H % Hkv == 0;
  for (int i = 0; i < 4; ++i) same = same && k.shape[i] == v.shape[i];
  if (!same || q.fmt != k.fmt || (v.fmt != FP4ATTN_FMT_MXFP4 && v.fmt != kFmtE4m3))
    return assertion("K and V must have one shape, Q the same but for the heads, whose number K's divides; Q and K one format, V MXFP4 or E4M3");
  if (q.per_head != k.per_head) return assertion("Q and K must both carry per-head factors, or neither");
  const bool fp8 = v.fmt == kFmtE4m3;
  PyObject* const seq = args[14];
  if (seq != Py_None) {
    if (!THPVariable_Check(seq)) return assertion("seq_len must be a contiguous CUDA int32 tensor of B counts");
    const at::Tensor& t = THPVariable_Unpack(seq);
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.numel() != B || !t.is_contiguous())
      return assertion("seq_len must be a contiguous CUDA int32 tensor of B counts");
  }
  fp4attn_operands ops = {};
  ops.q = q.packed; ops.k = k.packed; ops.v = v.packed;
  ops.q_sf = q.scales; ops.k_sf = k.scales; ops.v_sf = fp8 ? nullptr : v.scales;
  ops.q_G = (const float*)q.G; ops.k_G = (const float*)k.G;
  ops.qk_fmt = q.fmt;
  ops.kv_heads = Hkv;
  ops.g_per_head = q.per_head ? 1 : 0;
  ops.pv_fmt = fp8 ? FP4ATTN_PV_E4M3 : FP4ATTN_PV_MXFP4;
  ops.v_G = fp8 ? (const float*)v.G : nullptr;
  void *seq_len, *out_ptr, *lse_ptr, *status;
  if (!number(args[3], &ops.softmax_scale) || !number(args[8], &ops.affine_a) || !number(args[9], &ops.affine_b) ||
      !ints(args + 7, 1, &ops.p_map, true) || !ints(args + 10, 1, &ops.p_scale_rule, true) ||
      !ints(args + 12, 1, &ops.exact_pairs, true) || !ints(args + 13, 1, &ops.schedule, true) || !data_of(seq, &seq_len) ||
      !data_of(args[4], &out_ptr) || !data_of(args[5], &lse_ptr) || !data_of(args[6], &status))
    return nullptr;
  if ((ops.causal = PyObject_IsTrue(args[11])) < 0) return nullptr;
  ops.seq_len = (const int*)seq_len;
  if (args[15] != Py_None) {
    ops.row_reference = FP4ATTN_REFERENCE_FIXED;
    if (!ints(args + 15, 1, &ops.fixed_reference, true)) return nullptr;
  }
  THPObjectPtr out(Py_NewRef(args[4])), lse(Py_NewRef(args[5]));        // given back on every way out, an exception's too
  if (out.get() == Py_None || lse.get() == Py_None) {
    Results r;
    at::Tensor none, &o = out.get() == Py_None ? r.add({B, H, N, d}, at::kBFloat16) : none, &l = lse.get() == Py_None ? r.add({B, H, N}, at::kFloat) : none;
    r.allocate(q.device);
    if (o.defined()) { out_ptr = o.data_ptr(); out = THPVariable_Wrap(o); }
    if (l.defined()) { lse_ptr = l.data_ptr(); lse = THPVariable_Wrap(l); }
    if (!out || !lse) return nullptr;
  }
  const int rc = unlocked([&] { return g_api.fwd(&ops, B, H, N, d, out_ptr, (float*)lse_ptr, (int*)status, stream()); });
  if (rc) return fail(rc, "fp4attn_fwd");
  return Py_BuildValue("(NN)", out.release(), lse.release());
  FP4_CATCH
}

// ---------------------------------------------------------------- serving: positions, cache, attention over it

// A tensor [B, heads, N, d] on a CUDA device, the last axis contiguous
struct Strided {
  const at::Tensor* t = nullptr;
  int B = 0, H = 0, N = 0, d = 0, type = -1;
  bool empty = false;                                    // (then refused, for this reason)
  fp4attn_view view{};
  bool take(PyObject* o, bool fp32) {
    if (!THPVariable_Check(o)) return false;
    t = &THPVariable_Unpack(o);
    if (!t->is_cuda() || t->dim() != 4) return false;
    type = t->scalar_type() == at::kBFloat16 ? FP4ATTN_TYPE_BF16 : t->scalar_type() == at::kHalf ? FP4ATTN_TYPE_FP16
         : t->scalar_type() == at::kFloat && fp32 ? FP4ATTN_TYPE_FP32 : -1;
    const auto s = t->sizes(), st = t->strides();
    empty = type >= 0 && t->numel() == 0;
    for (int i = 0; i < 4; ++i)
      if (s[i] > INT32_MAX || s[i] < 1) return false;
    B = (int)s[0]; H = (int)s[1]; N = (int)s[2]; d = (int)s[3];
    // an axis of one index may have any stride: it is never taken, and must not spoil the alignment
    view = {t->data_ptr(), B > 1 ? st[0] : 0, H > 1 ? st[1] : 0, N > 1 ? st[2] : 0};
    return type >= 0 && (d == 1 || st[3] == 1);
  }
  bool like(const Strided& o) const { return B == o.B && N == o.N && d == o.d && type == o.type && t->device() == o.t->device(); }
  bool begins_with(const Strided& o) const { return t && o.t && view.data == o.view.data; }
  bool same_view(const Strided& o) const {
    return begins_with(o) && H == o.H && view.stride_b == o.view.stride_b && view.stride_h == o.view.stride_h && view.stride_n == o.view.stride_n;
  }
  // no two elements at one address (what is written must not be a broadcast)
  bool distinct() const { return t->is_non_overlapping_and_dense() || spread(); }

 private:
  bool spread() const {
    // strides sorted: each at least as long as what the smaller ones span
    int64_t size[3] = {B, H, N}, stride[3] = {view.stride_b, view.stride_h, view.stride_n}, span = d;
    for (int k = 0; k < 3; ++k) {
      int at = -1;
      for (int i = 0; i < 3; ++i)
        if (size[i] > 1 && (at < 0 || stride[i] < stride[at])) at = i;
      if (at < 0) break;
      if (stride[at] < span) return false;
      span = stride[at] * (size[at] - 1) + span;
      size[at] = 1;
    }
    return true;
  }
};
const char* kNothing = "a call needs at least one sequence, head, token and element: leave out calls of an empty batch";
// the shape `sizes`, or None
bool shaped(PyObject* o, at::IntArrayRef sizes) { return o == Py_None || (THPVariable_Check(o) && THPVariable_Unpack(o).sizes() == sizes); }
// a contiguous tensor of `n` values of `type` on `device`, or None where that is allowed
bool plain(PyObject* o, at::ScalarType type, int64_t n, c10::Device device, bool optional, void** ptr) {
  *ptr = nullptr;
  if (o == Py_None) return optional;
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || t.numel() != n || !t.is_contiguous() || t.device() != device) return false;
  *ptr = t.data_ptr();
  return true;
}

struct Cache {
  fp4attn_cache c{};
  c10::Device device{c10::kCPU};
  const char* take(PyObject* o) {                        // null, or what is wrong ("": an exception is set)
    PyObject* v[C_COUNT] = {};
    const char* wrong = nullptr;
    for (int i = 0; i < C_COUNT && !wrong; ++i)
      if (!(v[i] = PyObject_GetAttr(o, g_cache_names[i]))) wrong = "";
    if (!wrong) wrong = read(v);
    for (int i = 0; i < C_COUNT; ++i) Py_XDECREF(v[i]);
    return wrong;
  }

 private:
  const char* read(PyObject** v) {
    if (!THPVariable_Check(v[C_PAGES])) return "cache.pages must be a contiguous CUDA uint8 tensor [pages, KV heads, bytes of a record]";
    const at::Tensor& t = THPVariable_Unpack(v[C_PAGES]);
    if (!t.is_cuda() || t.scalar_type() != at::kByte || t.dim() != 3 || !t.is_contiguous() || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX)
      return "cache.pages must be a contiguous CUDA uint8 tensor [pages, KV heads, bytes of a record]";
    int a[3];
    if (!ints(v + C_FMT, 3, a)) return "";
    c.pages = t.data_ptr();
    device = t.device();
    c.num_pages = (int)t.size(0); c.kv_heads = (int)t.size(1);
    c.fmt = a[0]; c.page_size = a[1]; c.d = a[2];
    const size_t record = g_api.cache_record_bytes(c.fmt, c.page_size, c.d);
    if (record && (size_t)t.size(2) != record) return "cache.pages must have fp4attn_cache_record_bytes(fmt, page_size, d) bytes a record";
    void *kg, *vg;
    if (!plain(v[C_K_G], at::kFloat, c.kv_heads, device, false, &kg) || !plain(v[C_V_G], at::kFloat, c.kv_heads, device, false, &vg))
      return "cache.k_G and cache.v_G must be contiguous CUDA float32 tensors with one factor per KV head";
    c.k_G = (const float*)kg; c.v_G = (const float*)vg;
    return nullptr;
  }
};
// what the calls over a cache share: table, counts
struct Batch {
  const int *table = nullptr, *start = nullptr, *count = nullptr;
  int max_pages = 0;
  int* status = nullptr;
  const char* take(int B, c10::Device device, PyObject* table_o, PyObject* start_o, PyObject* count_o, PyObject* status_o) {
    if (!THPVariable_Check(table_o)) return "block_table must be a contiguous CUDA int32 tensor [B, pages of a sequence]";
    const at::Tensor& t = THPVariable_Unpack(table_o);
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != 2 || !t.is_contiguous() || t.size(0) != B || t.size(1) < 1 ||
        t.size(1) > INT32_MAX || t.device() != device)
      return "block_table must be a contiguous CUDA int32 tensor [B, pages of a sequence] on the cache's device";
    table = t.data_ptr<int>();
    max_pages = (int)t.size(1);
    void *s, *c, *st;
    if (!plain(start_o, at::kInt, B, device, false, &s)) return "start / context must be a contiguous CUDA int32 tensor of B positions on the cache's device";
    if (!plain(count_o, at::kInt, B, device, true, &c)) return "count must be a contiguous CUDA int32 tensor of B counts on the cache's device";
    if (!plain(status_o, at::kInt, 1, device, true, &st)) return "status must be a CUDA int32 tensor of one element on the cache's device";
    start = (const int*)s; count = (const int*)c; status = (int*)st;
    return nullptr;
  }
};
// Output tensors: what the caller gave, checked, or pieces of one allocation
struct Outputs {
  Results r;
  at::Tensor* own[2] = {nullptr, nullptr};
  bool take(int i, PyObject* o, const Strided& like, Strided* out) {
    if (o != Py_None) return out->take(o, true) && out->like(like) && out->H == like.H && out->distinct();
    own[i] = &r.add({like.B, like.H, like.N, like.d}, like.t->scalar_type());
    return true;
  }
  void allocate(c10::Device device, Strided* out) {
    if (r.n) r.allocate(device);
    for (int i = 0; i < 2; ++i)
      if (own[i]) out[i].view = {own[i]->data_ptr(), own[i]->stride(0), own[i]->stride(1), own[i]->stride(2)};
  }
  PyObject* give(int i, PyObject* o) const { return own[i] ? THPVariable_Wrap(*own[i]) : Py_NewRef(o); }
};

// rotary(q, k, positions, inv_freq, interleaved, transposed, factor, q_out, k_out) -> q_out, or (q_out, k_out); NotImplemented, with nothing done,
// where gradients are recorded and an input takes one: binding.py then makes the call inside an autograd function
PyObject* py_rotary(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 9) return assertion("rotary takes 9 arguments");
  Strided x[2], y[2];
  Outputs outputs;
  const bool two = args[1] != Py_None;
  if (!x[0].take(args[0], true) || (two && !(x[1].take(args[1], true) && x[1].like(x[0]))))
    return assertion(x[0].empty || x[1].empty ? kNothing : "q (and k) must be CUDA tensors [B, heads, N, d], bfloat16, float16 or float32, the last axis contiguous; k of q's B, N, d, type and device");
  if (!two && args[8] != Py_None) return assertion("k_out is given but k is not");
  const c10::Device device = x[0].t->device();
  void *positions, *freq = nullptr;
  if (!plain(args[2], at::kInt, (int64_t)x[0].B * x[0].N, device, false, &positions) || !shaped(args[2], {x[0].B, x[0].N}))
    return assertion("positions must be a contiguous CUDA int32 tensor [B, N] on q's device");
  const int64_t pairs = THPVariable_Check(args[3]) ? THPVariable_Unpack(args[3]).numel() : 0;
  if (pairs < 1 || pairs > INT32_MAX / 2 || !plain(args[3], at::kFloat, pairs, device, false, &freq))
    return assertion("inv_freq must be a contiguous CUDA float32 tensor with one frequency per pair on q's device");
  float factor;
  const int interleaved = PyObject_IsTrue(args[4]), transposed = PyObject_IsTrue(args[5]);
  if (interleaved < 0 || transposed < 0 || !number(args[6], &factor)) return nullptr;
  if (c10::GradMode::is_enabled()) {
    if (THPVariable_Unpack(args[3]).requires_grad()) return assertion("inv_freq takes no gradient");
    if (x[0].t->requires_grad() || (two && x[1].t->requires_grad())) {
      if (args[7] != Py_None || args[8] != Py_None)
        return assertion("q_out and k_out carry no gradient, and an input requires one: leave them out, or call under torch.no_grad()");
      Py_RETURN_NOTIMPLEMENTED;
    }
  }
  const c10::cuda::OptionalCUDAGuard guard(device);
  for (int i = 0; i <= (int)two; ++i)
    if (!outputs.take(i, args[7 + i], x[i], &y[i]))
      return assertion("an output must be a CUDA tensor of its input's shape, type and device, the last axis contiguous, no element twice");
  // What is written in place is written by the thread that has read it; in another order, or over the other tensor, it is not
  for (int i = 0; i <= (int)two; ++i)
    if ((y[i].begins_with(x[i]) && !y[i].same_view(x[i])) || y[i].begins_with(x[1 - i]) || (i == 1 && y[1].begins_with(y[0])))
      return assertion("an output may be its own input, the same view of it, and must not overlap any other tensor of the call");
  outputs.allocate(device, y);
  const int rc = unlocked([&] {
    return g_api.rotary(&x[0].view, two ? &x[1].view : nullptr, &y[0].view, two ? &y[1].view : nullptr, x[0].type, x[0].B, x[0].H, x[1].H,
                        x[0].N, x[0].d, (const int*)positions, (const float*)freq, (int)pairs, interleaved, transposed, factor, stream());
  });
  if (rc) return fail(rc, "fp4attn_rotary");
  if (!two) return outputs.give(0, args[7]);
  return Py_BuildValue("(NN)", outputs.give(0, args[7]), outputs.give(1, args[8]));
  FP4_CATCH
}

// cache_write(cache, k, v, block_table, start, count, positions, inv_freq, interleaved, factor, status)
PyObject* py_cache_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 11) return assertion("cache_write takes 11 arguments");
  Cache cache;
  if (const char* wrong = cache.take(args[0])) return *wrong ? assertion(wrong) : nullptr;
  Strided k, v;
  if (!k.take(args[1], false) || !v.take(args[2], false) || !v.like(k) || v.H != k.H || k.H != cache.c.kv_heads || k.d != cache.c.d ||
      k.t->device() != cache.device)
    return assertion(k.empty || v.empty ? kNothing : "k and v must be CUDA tensors [B, KV heads, N, d] of the cache's heads, d and device, bfloat16 or float16, the last axis contiguous");
  Batch batch;
  if (const char* wrong = batch.take(k.B, cache.device, args[3], args[4], args[5], args[10])) return assertion(wrong);
  void *positions, *freq = nullptr;
  if (!plain(args[6], at::kInt, (int64_t)k.B * k.N, cache.device, true, &positions) || !shaped(args[6], {k.B, k.N}))
    return assertion("positions must be a contiguous CUDA int32 tensor [B, N] on the cache's device");
  int64_t pairs = 0;
  if (args[7] != Py_None) {
    pairs = THPVariable_Check(args[7]) ? THPVariable_Unpack(args[7]).numel() : 0;
    if (pairs < 1 || pairs > INT32_MAX / 2 || !plain(args[7], at::kFloat, pairs, cache.device, false, &freq))
      return assertion("inv_freq must be a contiguous CUDA float32 tensor with one frequency per pair on the cache's device");
  } else if (positions) {
    return assertion("positions are given but inv_freq is not");
  }
  float factor;
  const int interleaved = PyObject_IsTrue(args[8]);
  if (interleaved < 0 || !number(args[9], &factor)) return nullptr;
  const c10::cuda::OptionalCUDAGuard guard(cache.device);
  const int rc = unlocked([&] {
    return g_api.cache_write(&cache.c, &k.view, &v.view, k.type, k.B, k.N, batch.table, batch.max_pages, batch.start, batch.count,
                             (const int*)positions, (const float*)freq, (int)pairs, interleaved, factor, batch.status, stream());
  });
  if (rc) return fail(rc, "fp4attn_cache_write");
  Py_RETURN_NONE;
  FP4_CATCH
}

// cache_read(cache, block_table, start, N, count, is float16, k_out, v_out, status) -> (k_out, v_out)
PyObject* py_cache_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 9) return assertion("cache_read takes 9 arguments");
  Cache cache;
  if (const char* wrong = cache.take(args[0])) return *wrong ? assertion(wrong) : nullptr;
  if (!THPVariable_Check(args[1]) || THPVariable_Unpack(args[1]).dim() != 2)
    return assertion("block_table must be a contiguous CUDA int32 tensor [B, pages of a sequence]");
  const int64_t B = THPVariable_Unpack(args[1]).size(0);
  int N;
  if (!ints(args + 3, 1, &N)) return nullptr;
  const int half = PyObject_IsTrue(args[5]);
  if (half < 0) return nullptr;
  if (B < 1 || B > INT32_MAX || N < 1) return assertion(kNothing);
  Batch batch;
  if (const char* wrong = batch.take((int)B, cache.device, args[1], args[2], args[4], args[8])) return assertion(wrong);
  const c10::cuda::OptionalCUDAGuard guard(cache.device);
  const at::ScalarType type = half ? at::kHalf : at::kBFloat16;
  Strided out[2];
  Outputs outputs;
  for (int i = 0; i < 2; ++i) {
    if (args[6 + i] == Py_None) {
      outputs.own[i] = &outputs.r.add({B, cache.c.kv_heads, N, cache.c.d}, type);
    } else if (!out[i].take(args[6 + i], false) || out[i].t->scalar_type() != type || out[i].B != B || out[i].H != cache.c.kv_heads ||
               out[i].N != N || out[i].d != cache.c.d || out[i].t->device() != cache.device || !out[i].distinct()) {
      return assertion("k_out and v_out must be CUDA tensors [B, KV heads, N, d] of the cache's heads, d and device and of dtype, the last axis contiguous, no element twice");
    }
  }
  if (out[1].begins_with(out[0])) return assertion("k_out and v_out must not overlap");
  outputs.allocate(cache.device, out);
  for (at::Tensor* own : outputs.own)
    if (own && batch.count) own->zero_();                // rows behind the counts are not written
  const int rc = unlocked([&] {
    return g_api.cache_read(&cache.c, &out[0].view, &out[1].view, half ? FP4ATTN_TYPE_FP16 : FP4ATTN_TYPE_BF16, (int)B, N, batch.table,
                            batch.max_pages, batch.start, batch.count, batch.status, stream());
  });
  if (rc) return fail(rc, "fp4attn_cache_read");
  return Py_BuildValue("(NN)", outputs.give(0, args[6]), outputs.give(1, args[7]));
  FP4_CATCH
}

// tree_attention(q, cache, block_table, context, tree_mask, count, softmax_scale, out, lse, status) -> (out, lse)
PyObject* py_tree_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 10) return assertion("tree_attention takes 10 arguments");
  Cache cache;
  if (const char* wrong = cache.take(args[1])) return *wrong ? assertion(wrong) : nullptr;
  Strided q;
  if (!q.take(args[0], false) || q.d != cache.c.d || q.t->device() != cache.device || cache.c.kv_heads < 1 || q.H % cache.c.kv_heads != 0)
    return assertion(q.empty ? kNothing : "q must be a CUDA tensor [B, H, T, d] of the cache's d and device, bfloat16 or float16, the last axis contiguous; H a multiple of the KV heads");
  Batch batch;
  if (const char* wrong = batch.take(q.B, cache.device, args[2], args[3], args[5], args[9])) return assertion(wrong);
  void *mask, *out_ptr, *lse_ptr;
  if (!plain(args[4], at::kLong, (int64_t)q.B * q.N, cache.device, true, &mask) || !shaped(args[4], {q.B, q.N}))
    return assertion("tree_mask must be a contiguous CUDA int64 tensor [B, T] on the cache's device");
  float scale;
  if (!number(args[6], &scale)) return nullptr;
  const int64_t rows = (int64_t)q.B * q.H * q.N;
  if (!plain(args[7], q.t->scalar_type(), rows * q.d, cache.device, true, &out_ptr) || !shaped(args[7], {q.B, q.H, q.N, q.d}) ||
      !plain(args[8], at::kFloat, rows, cache.device, true, &lse_ptr) || !shaped(args[8], {q.B, q.H, q.N}))
    return assertion("out [B, H, T, d] of q's type and lse [B, H, T] float32 must be contiguous CUDA tensors on the cache's device");
  const c10::cuda::OptionalCUDAGuard guard(cache.device);
  const size_t nw = g_api.tree_workspace_bytes(q.B, q.H, cache.c.kv_heads, q.N, q.d);
  THPObjectPtr out(Py_NewRef(args[7])), lse(Py_NewRef(args[8]));
  Results r;
  at::Tensor none, &o = out_ptr ? none : r.add({q.B, q.H, q.N, q.d}, q.t->scalar_type()), &l = lse_ptr ? none : r.add({q.B, q.H, q.N}, at::kFloat);
  if (r.n) r.allocate(cache.device);
  const at::Tensor ws = nw ? device_empty({(int64_t)nw}, at::kByte, cache.device) : none;
  if (o.defined()) {
    if (batch.count) o.zero_();                          // rows behind the counts are not written
    out_ptr = o.data_ptr();
    out = THPVariable_Wrap(o);
  }
  if (l.defined()) {
    if (batch.count) l.fill_(-std::numeric_limits<float>::infinity());
    lse_ptr = l.data_ptr();
    lse = THPVariable_Wrap(l);
  }
  if (!out || !lse) return nullptr;
  const int rc = unlocked([&] {
    return g_api.tree_attention(&q.view, q.type, &cache.c, q.B, q.H, q.N, batch.table, batch.max_pages, batch.start, batch.count,
                                (const unsigned long long*)mask, scale, out_ptr, (float*)lse_ptr, batch.status,
                                nw ? ws.data_ptr() : nullptr, nw, stream());
  });
  if (rc) return fail(rc, "fp4attn_tree_attention");
  return Py_BuildValue("(NN)", out.release(), lse.release());
  FP4_CATCH
}

// ---------------------------------------------------------------- prompts and shared prefixes over the cache

// What attention over a cache takes besides its masks, and what it gives: checks, outputs, workspace
struct Attention {
  Cache cache;
  Strided q;
  Batch batch;
  float scale = 0.f, cap = 0.f;
  void *slopes = nullptr, *out_ptr = nullptr, *lse_ptr = nullptr;
  THPObjectPtr out, lse;
  at::Tensor ws;
  size_t nw = 0;
  // null, or what is wrong ("": an exception is set)
  const char* take(PyObject* q_o, PyObject* cache_o, PyObject* table, PyObject* context, PyObject* count, PyObject* scale_o, PyObject* cap_o,
                   PyObject* slopes_o, PyObject* out_o, PyObject* lse_o, PyObject* status) {
    if (const char* wrong = cache.take(cache_o)) return wrong;
    if (!q.take(q_o, false) || q.d != cache.c.d || q.t->device() != cache.device || cache.c.kv_heads < 1 || q.H % cache.c.kv_heads != 0)
      return q.empty ? kNothing : "q must be a CUDA tensor [B, H, T, d] of the cache's d and device, bfloat16 or float16, the last axis contiguous; H a multiple of the KV heads";
    if (const char* wrong = batch.take(q.B, cache.device, table, context, count, status)) return wrong;
    if (!number(scale_o, &scale) || !number(cap_o, &cap)) return "";
    if (!plain(slopes_o, at::kFloat, q.H, cache.device, true, &slopes)) return "slopes must be a contiguous CUDA float32 tensor [H] on the cache's device";
    const int64_t rows = (int64_t)q.B * q.H * q.N;
    if (!plain(out_o, q.t->scalar_type(), rows * q.d, cache.device, true, &out_ptr) || !shaped(out_o, {q.B, q.H, q.N, q.d}) ||
        !plain(lse_o, at::kFloat, rows, cache.device, true, &lse_ptr) || !shaped(lse_o, {q.B, q.H, q.N}))
      return "out [B, H, T, d] of q's type and lse [B, H, T] float32 must be contiguous CUDA tensors on the cache's device";
    if (overlaps(out_o, lse_o, rows)) return "out may be q, the same view of it; otherwise out, lse and q must not overlap";
    if (c10::GradMode::is_enabled() && (q.t->requires_grad() || (slopes && THPVariable_Unpack(slopes_o).requires_grad())))
      return "attention over a quantized cache takes no gradient: detach the inputs, or call under torch.no_grad()";
    return nullptr;
  }
  // false: an exception is set
  bool allocate(PyObject* out_o, PyObject* lse_o, size_t bytes) {
    nw = bytes;
    out = THPObjectPtr(Py_NewRef(out_o));
    lse = THPObjectPtr(Py_NewRef(lse_o));
    Results r;
    at::Tensor none, &o = out_ptr ? none : r.add({q.B, q.H, q.N, q.d}, q.t->scalar_type()), &l = lse_ptr ? none : r.add({q.B, q.H, q.N}, at::kFloat);
    if (r.n) r.allocate(cache.device);
    if (nw) ws = device_empty({(int64_t)nw}, at::kByte, cache.device);
    if (o.defined()) {
      if (batch.count) o.zero_();                        // rows behind the counts are not written
      out_ptr = o.data_ptr();
      out = THPVariable_Wrap(o);
    }
    if (l.defined()) {
      if (batch.count) l.fill_(-std::numeric_limits<float>::infinity());
      lse_ptr = l.data_ptr();
      lse = THPVariable_Wrap(l);
    }
    return out && lse;
  }
  void* workspace() const { return nw ? ws.data_ptr() : nullptr; }
  PyObject* give() { return Py_BuildValue("(NN)", out.release(), lse.release()); }

 private:
  // Tensors of the caller's over one another.  A row's Q has been read when its O is written, so O may lie where Q does; nothing else may: other
  // rows' Q, or both outputs of a row, in one place.  (Of a q with gaps only the beginning is looked at: what lies in the gaps is not q.)
  bool overlaps(PyObject* out_o, PyObject* lse_o, int64_t rows) const {
    const auto meet = [](const void* a, int64_t na, const void* b, int64_t nb) {
      return a && b && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
    };
    const int64_t out_bytes = rows * q.d * 2, q_bytes = q.t->is_non_overlapping_and_dense() ? out_bytes : 1;
    Strided o;
    const bool in_place = out_ptr && o.take(out_o, false) && o.same_view(q);
    return meet(out_ptr, out_bytes, lse_ptr, rows * 4) || meet(lse_ptr, rows * 4, q.view.data, q_bytes) ||
           (!in_place && meet(out_ptr, out_bytes, q.view.data, q_bytes));
  }
};

// paged_attention(q, cache, block_table, context, count, first, last, softmax_scale, soft_cap, slopes, out, lse, status) -> (out, lse)
PyObject* py_paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 13) return assertion("paged_attention takes 13 arguments");
  Attention a;
  if (const char* wrong = a.take(args[0], args[1], args[2], args[3], args[4], args[7], args[8], args[9], args[10], args[11], args[12]))
    return *wrong ? assertion(wrong) : nullptr;
  const Strided& q = a.q;
  void *first, *last;
  if (!plain(args[5], at::kInt, (int64_t)q.B * q.N, a.cache.device, true, &first) || !shaped(args[5], {q.B, q.N}) ||
      !plain(args[6], at::kInt, (int64_t)q.B * q.N, a.cache.device, true, &last) || !shaped(args[6], {q.B, q.N}))
    return assertion("first and last must be contiguous CUDA int32 tensors [B, T] on the cache's device");
  const c10::cuda::OptionalCUDAGuard guard(a.cache.device);
  if (!a.allocate(args[10], args[11], g_api.paged_workspace_bytes(q.B, q.H, a.cache.c.kv_heads, q.N, q.d))) return nullptr;
  const int rc = unlocked([&] {
    return g_api.paged_attention(&q.view, q.type, &a.cache.c, q.B, q.H, q.N, a.batch.table, a.batch.max_pages, a.batch.start, a.batch.count,
                                 (const int*)first, (const int*)last, a.scale, a.cap, (const float*)a.slopes, a.out_ptr, (float*)a.lse_ptr,
                                 a.batch.status, a.workspace(), a.nw, stream());
  });
  if (rc) return fail(rc, "fp4attn_paged_attention");
  return a.give();
  FP4_CATCH
}

// shared_prefix_attention(q, cache, prefix_table, prefix_length, group_start, block_table, context, tree_mask, count, softmax_scale, soft_cap,
//                         slopes, out, lse, status) -> (out, lse)
PyObject* py_shared_prefix_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 15) return assertion("shared_prefix_attention takes 15 arguments");
  Attention a;
  if (const char* wrong = a.take(args[0], args[1], args[5], args[6], args[8], args[9], args[10], args[11], args[12], args[13], args[14]))
    return *wrong ? assertion(wrong) : nullptr;
  const Strided& q = a.q;
  const char* const prefix_rule = "prefix_table must be a contiguous CUDA int32 tensor [groups, pages of a prefix] on the cache's device";
  if (!THPVariable_Check(args[2]) || THPVariable_Unpack(args[2]).dim() != 2) return assertion(prefix_rule);
  const int64_t groups = THPVariable_Unpack(args[2]).size(0), pages = THPVariable_Unpack(args[2]).size(1);
  void *table, *length, *start, *mask;
  if (groups < 1 || pages < 1 || groups > INT32_MAX || pages > INT32_MAX || !plain(args[2], at::kInt, groups * pages, a.cache.device, false, &table))
    return assertion(prefix_rule);
  if (!plain(args[3], at::kInt, groups, a.cache.device, false, &length)) return assertion("prefix_length must be a contiguous CUDA int32 tensor of one length per group on the cache's device");
  if (!plain(args[4], at::kInt, groups + 1, a.cache.device, false, &start)) return assertion("group_start must be a contiguous CUDA int32 tensor of groups + 1 entries on the cache's device");
  if (!plain(args[7], at::kLong, (int64_t)q.B * q.N, a.cache.device, true, &mask) || !shaped(args[7], {q.B, q.N}))
    return assertion("tree_mask must be a contiguous CUDA int64 tensor [B, T] on the cache's device");
  const c10::cuda::OptionalCUDAGuard guard(a.cache.device);
  if (!a.allocate(args[12], args[13], g_api.shared_workspace_bytes(q.B, q.H, a.cache.c.kv_heads, q.N, q.d, (int)groups))) return nullptr;
  const int rc = unlocked([&] {
    return g_api.shared_prefix_attention(&q.view, q.type, &a.cache.c, q.B, q.H, q.N, (int)groups, (const int*)table, (int)pages, (const int*)length,
                                         (const int*)start, a.batch.table, a.batch.max_pages, a.batch.start, a.batch.count,
                                         (const unsigned long long*)mask, a.scale, a.cap, (const float*)a.slopes, a.out_ptr, (float*)a.lse_ptr,
                                         a.batch.status, a.workspace(), a.nw, stream());
  });
  if (rc) return fail(rc, "fp4attn_shared_prefix_attention");
  return a.give();
  FP4_CATCH
}

// ---------------------------------------------------------------- pages out of a pool

struct Pool {
  fp4attn_page_pool c{};
  c10::Device device{c10::kCPU};
  const char* take(PyObject* o) {                        // null, or what is wrong ("": an exception is set)
    PyObject* v[P_COUNT] = {};
    const char* wrong = nullptr;
    for (int i = 0; i < P_COUNT && !wrong; ++i)
      if (!(v[i] = PyObject_GetAttr(o, g_pool_names[i]))) wrong = "";
    if (!wrong) wrong = read(v);
    for (int i = 0; i < P_COUNT; ++i) Py_XDECREF(v[i]);
    return wrong;
  }

 private:
  const char* read(PyObject** v) {
    const char* const rule = "pool.free must be a contiguous CUDA int32 tensor of page numbers, pool.count and pool.turn int32 tensors of one element on its device";
    if (!THPVariable_Check(v[P_FREE])) return rule;
    const at::Tensor& t = THPVariable_Unpack(v[P_FREE]);
    device = t.device();
    void *free, *count, *turn;
    if (t.numel() < 1 || t.numel() > INT32_MAX || !plain(v[P_FREE], at::kInt, t.numel(), device, false, &free) ||
        !plain(v[P_COUNT_OF], at::kInt, 1, device, false, &count) || !plain(v[P_TURN], at::kInt, 1, device, false, &turn))
      return rule;
    if (!ints(v + P_PAGE_SIZE, 1, &c.page_size)) return "";
    c.free = (int*)free; c.count = (int*)count; c.turn = (int*)turn;
    c.num_pages = (int)t.numel();
    return nullptr;
  }
};

// block_table, which is written
const char* take_table(PyObject* o, c10::Device device, int** table, int* B, int* max_pages) {
  const char* const rule = "block_table must be a contiguous CUDA int32 tensor [B, pages of a sequence] on the pool's device";
  if (!THPVariable_Check(o)) return rule;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != 2 || !t.is_cuda() || t.scalar_type() != at::kInt || !t.is_contiguous() || t.device() != device) return rule;
  if (t.size(0) < 1 || t.size(0) > INT32_MAX) return kNothing;
  if (t.size(1) < 1 || t.size(1) > INT32_MAX) return rule;
  *table = t.data_ptr<int>();
  *B = (int)t.size(0);
  *max_pages = (int)t.size(1);
  return nullptr;
}

// pages_assign(pool, block_table, start, count, N, status) -> (slots, positions), or (None, None) with N = 0
PyObject* py_pages_assign(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 6) return assertion("pages_assign takes 6 arguments");
  Pool pool;
  if (const char* wrong = pool.take(args[0])) return *wrong ? assertion(wrong) : nullptr;
  int *table, B, max_pages, N;
  if (const char* wrong = take_table(args[1], pool.device, &table, &B, &max_pages)) return assertion(wrong);
  if (!ints(args + 4, 1, &N)) return nullptr;
  if (N < 0 || (N == 0 && args[3] == Py_None)) return assertion("N must be a number of tokens; it may be 0 where count is given");
  void *start, *count, *status;
  if (!plain(args[2], at::kInt, B, pool.device, false, &start) || !plain(args[3], at::kInt, B, pool.device, true, &count))
    return assertion("start and count must be contiguous CUDA int32 tensors of B values on the pool's device");
  if (!plain(args[5], at::kInt, 1, pool.device, true, &status)) return assertion("status must be a CUDA int32 tensor of one element on the pool's device");
  const c10::cuda::OptionalCUDAGuard guard(pool.device);
  Results r;
  at::Tensor none, &slots = N ? r.add({B, N}, at::kLong) : none, &positions = N ? r.add({B, N}, at::kInt) : none;
  if (N) r.allocate(pool.device);
  const int rc = unlocked([&] {
    return g_api.pages_assign(&pool.c, B, N, table, max_pages, (const int*)start, (const int*)count, N ? (long long*)slots.data_ptr() : nullptr,
                              N ? positions.data_ptr<int>() : nullptr, (int*)status, stream());
  });
  if (rc) return fail(rc, "fp4attn_pages_assign");
  if (!N) return Py_BuildValue("(OO)", Py_None, Py_None);
  return Py_BuildValue("(NN)", THPVariable_Wrap(slots), THPVariable_Wrap(positions));
  FP4_CATCH
}

// pages_release(pool, block_table, length, keep, status)
PyObject* py_pages_release(PyObject*, PyObject* const* args, Py_ssize_t n) {
  FP4_TRY
  if (n != 5) return assertion("pages_release takes 5 arguments");
  Pool pool;
  if (const char* wrong = pool.take(args[0])) return *wrong ? assertion(wrong) : nullptr;
  int *table, B, max_pages;
  if (const char* wrong = take_table(args[1], pool.device, &table, &B, &max_pages)) return assertion(wrong);
  void *length, *keep, *status;
  if (!plain(args[2], at::kInt, B, pool.device, false, &length) || !plain(args[3], at::kInt, B, pool.device, true, &keep))
    return assertion("length and keep must be contiguous CUDA int32 tensors of B values on the pool's device");
  if (!plain(args[4], at::kInt, 1, pool.device, true, &status)) return assertion("status must be a CUDA int32 tensor of one element on the pool's device");
  const c10::cuda::OptionalCUDAGuard guard(pool.device);
  const size_t nw = g_api.release_workspace_bytes(B);
  at::Tensor ws;
  if (nw) ws = device_empty({(int64_t)nw}, at::kByte, pool.device);
  const int rc = unlocked([&] {
    return g_api.pages_release(&pool.c, B, table, max_pages, (const int*)length, (const int*)keep, (int*)status, nw ? ws.data_ptr() : nullptr, nw, stream());
  });
  if (rc) return fail(rc, "fp4attn_pages_release");
  Py_RETURN_NONE;
  FP4_CATCH
}

// init(error class, status_string, packed_bytes, ..., pages_release): addresses of the library's functions, in Api's order
PyObject* py_init(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t kFunctions = sizeof(Api) / sizeof(void*);
  if (n != 1 + kFunctions) return assertion("init takes the error class and one address per function");
  void* p[kFunctions];
  for (Py_ssize_t i = 0; i < kFunctions; ++i) {
    p[i] = PyLong_AsVoidPtr(args[1 + i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : assertion("a function's address is 0");
  }
  memcpy(static_cast<void*>(&g_api), p, sizeof p);
  Py_XSETREF(g_error, Py_NewRef(args[0]));
  Py_RETURN_NONE;
}

#define FP4_METHOD(NAME, FN) {NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(FN)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FP4_METHOD("init", py_init), FP4_METHOD("quantize", py_quantize), FP4_METHOD("quantize_mxfp4_rule", py_rule),
                         FP4_METHOD("quantize_nvfp4_per_head", py_per_head), FP4_METHOD("quantize_v_e4m3", py_e4m3),
                         FP4_METHOD("fwd", py_fwd), FP4_METHOD("rotary", py_rotary), FP4_METHOD("cache_write", py_cache_write),
                         FP4_METHOD("cache_read", py_cache_read), FP4_METHOD("tree_attention", py_tree_attention),
                         FP4_METHOD("paged_attention", py_paged_attention), FP4_METHOD("shared_prefix_attention", py_shared_prefix_attention),
                         FP4_METHOD("pages_assign", py_pages_assign), FP4_METHOD("pages_release", py_pages_release), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fp4attn_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__fp4attn_native() {
  const char* names[A_COUNT] = {"packed", "scales", "G", "fmt", "role", "shape", "per_head"};
  for (int i = 0; i < A_COUNT; ++i)
    if (!(g_names[i] = PyUnicode_InternFromString(names[i]))) return nullptr;
  const char* cache_names[C_COUNT] = {"pages", "k_G", "v_G", "fmt", "page_size", "d"};
  for (int i = 0; i < C_COUNT; ++i)
    if (!(g_cache_names[i] = PyUnicode_InternFromString(cache_names[i]))) return nullptr;
  const char* pool_names[P_COUNT] = {"free", "count", "turn", "page_size"};
  for (int i = 0; i < P_COUNT; ++i)
    if (!(g_pool_names[i] = PyUnicode_InternFromString(pool_names[i]))) return nullptr;
  return PyModule_Create(&module);
}
