// Argument marshalling of the Python binding in native code: tensors to zc_tensor4, the
// current HIP stream, a scratch buffer of the stream, and the call itself.  Nothing of the
// method happens here, and nothing about a call's tensors is kept.
//
// Why: a decode step at batch 1 is 9 us of GPU work, and describing its tensors through ctypes
// (attribute by attribute, a structure each) took 19 us of the caller's thread; here a tensor
// costs one look at its C++ object.  Steps of one 4096-token prompt issued one after the other:
// 18.5 -> 9.2 us each (the GPU's own time); six launches of a flush at batch 8: 47 -> 34 us.
//
// The library's entry points come in as addresses (bind), so that whichever build of the library
// the binding has loaded is the one that is called.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <map>
#include <mutex>
#include <tuple>
#include <utility>
#include <vector>

#include <ATen/ATen.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "zipcache.h"

namespace {

// ---- entry points, in the order of kNames ---------------------------------------------------
enum Fn {
  kProbe, kAccumulated, kPrefill, kSelect, kQuantize, kQuantizeKV, kDecode, kDecodeStatic, kProbs, kRows, kDequantize,
  kPagedTables, kPagedStore, kPagedLoad, kPagedAttention, kPagedShared, kPagedScores, kPagedEvict,
  kProbeWs, kQuantizeWs, kQuantizeKVWs, kDecodeWs, kPagedAttentionWs, kPagedSharedWs, kPagedEvictWs, kFnCount
};
const char* const kNames[kFnCount] = {
    "zc_probe_saliency", "zc_probe_accumulated", "zc_prefill_attention", "zc_select_salient", "zc_quantize_pack",
    "zc_quantize_pack_kv", "zc_decode_attention", "zc_decode_attention_static", "zc_decode_probs", "zc_rows_saliency",
    "zc_dequantize_cache", "zc_paged_tables", "zc_paged_store", "zc_paged_load", "zc_paged_attention", "zc_paged_shared_attention",
    "zc_paged_scores", "zc_paged_evict",
    "zc_probe_saliency_workspace", "zc_quantize_pack_workspace", "zc_quantize_pack_kv_workspace", "zc_decode_attention_workspace",
    "zc_paged_attention_workspace", "zc_paged_shared_attention_workspace", "zc_paged_evict_workspace"};
void* g_fn[kFnCount];

#define ZC_FN(id, name) reinterpret_cast<decltype(&name)>(g_fn[id])

// ---- arguments ---------------------------------------------------------------------------------
struct Bad {};   // a Python exception has been set

const at::Tensor& tensor_of(PyObject* o) {
  if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "expected a torch.Tensor, got %s", Py_TYPE(o)->tp_name); throw Bad(); }
  return THPVariable_Unpack(o);
}
void* ptr_of(PyObject* o) { return o == Py_None ? nullptr : tensor_of(o).data_ptr(); }
template <class T> T* ptr_as(PyObject* o) { return static_cast<T*>(ptr_of(o)); }

int64_t int_of(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Bad();
  return v;
}
float float_of(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Bad();
  return (float)v;
}

// A [B, H, L, D] tensor with unit stride on D; `row`: a [B, H, D] one stands for L = 1 too.
zc_tensor4 describe(PyObject* o, bool row = false) {
  const at::Tensor& t = tensor_of(o);
  const auto sz = t.sizes();
  const auto st = t.strides();
  const bool three = row && sz.size() == 3;
  if ((sz.size() != 4 && !three) || st.back() != 1) {
    PyErr_SetString(PyExc_AssertionError, "need a 4-D tensor with contiguous last axis");
    throw Bad();
  }
  zc_tensor4 r;
  r.ptr = t.data_ptr();
  switch (t.scalar_type()) {
    case at::kFloat: r.dtype = ZC_F32; break;
    case at::kHalf: r.dtype = ZC_F16; break;
    case at::kBFloat16: r.dtype = ZC_BF16; break;
    default: PyErr_Format(PyExc_KeyError, "%s", c10::toString(t.scalar_type())); throw Bad();
  }
  r.reserved = 0;
  r.B = sz[0]; r.H = sz[1]; r.sB = st[0]; r.sH = st[1];
  r.L = three ? 1 : sz[2];
  r.D = sz[three ? 2 : 3];
  r.sL = three ? r.D : st[2];
  return r;
}

// The zc_packed behind a ctypes structure, for the duration of a call.
struct Packed {
  Py_buffer view;
  explicit Packed(PyObject* o) {
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Bad();
    if (view.len != (Py_ssize_t)sizeof(zc_packed)) {
      PyBuffer_Release(&view);
      PyErr_SetString(PyExc_TypeError, "expected a zc_packed structure");
      throw Bad();
    }
  }
  Packed(const Packed&) = delete;
  ~Packed() { PyBuffer_Release(&view); }
  zc_packed* get() const { return static_cast<zc_packed*>(view.buf); }
};

// ---- scratch ---------------------------------------------------------------------------------
// One buffer per device, kind of call and stream (calls on different streams may run
// concurrently and must not share scratch memory), used by every call of that kind on that
// stream, in stream order.  A buffer is replaced by one at least half as large again and goes
// back to torch's allocator, which reuses it in the order of the stream - unless a call that used
// it was captured: the graph holds its address, and it is kept.  (So a stream holds less than one and a
// half times its largest request, and what its graphs were captured with.)  All of this runs
// under the interpreter lock; the launches do not, and a call is several of them: two threads' calls on
// one stream (by default all threads share one) would come between each other's.  So a call holds its buffer's mutex
// while it launches, taken when the interpreter lock has been given up and given back before that is taken again.
enum Kind { kScratchProbe, kScratchQuantize, kScratchQuantizeKV, kScratchDecode, kScratchPaged, kScratchShared, kScratchEvict };
struct Scratch { at::Tensor t; void* ptr = nullptr; size_t bytes = 0; bool captured = false; std::mutex* use = nullptr; };
std::map<std::tuple<int, int, void*>, Scratch>* g_scratch;
std::vector<at::Tensor>* g_captured;      // replaced buffers that graphs may hold
std::mutex g_static;                      // of the library's own buffer, zc_decode_attention_static's

// The reference keeps the buffer during the call, whose launch runs without the lock.
Scratch scratch(size_t need, const at::Tensor& like, Kind kind, hipStream_t stream) {
  Scratch& s = (*g_scratch)[std::make_tuple((int)like.device().index(), (int)kind, (void*)stream)];
  if (!s.use) s.use = new std::mutex;      // (as the buffers, until the process ends)
  if (!s.ptr || s.bytes < need) {
    size_t n = need < 256 ? 256 : need;
    if (s.ptr && n < s.bytes + s.bytes / 2) n = s.bytes + s.bytes / 2;
    at::Tensor t = at::zeros({(int64_t)n}, like.options().dtype(at::kByte));
    if (s.captured) g_captured->push_back(s.t);
    s.ptr = t.data_ptr();
    s.t = std::move(t);
    s.bytes = n;
    s.captured = false;
  }
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(stream, &status) != hipSuccess) {
    (void)hipGetLastError();
    s.captured = true;                     // (the default stream beside a capture: taken for one)
  }
  s.captured |= status != hipStreamCaptureStatusNone;
  return s;
}

hipStream_t current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Runs a call's launches without the interpreter lock (they may wait for room in the stream's queue), one call of those that
// share scratch memory (whose mutex is `use`, null: none) at a time.
template <class F> int unlocked(std::mutex* use, F&& f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  if (use) use->lock();
  rc = f();
  if (use) use->unlock();
  Py_END_ALLOW_THREADS
  return rc;
}
template <class F> int unlocked(F&& f) { return unlocked(nullptr, std::forward<F>(f)); }

// Every function below returns the library's status as an int (paged_tables: beside its outputs).
template <class F> PyObject* guarded(Fn id, Py_ssize_t n, Py_ssize_t want, F&& f) {
  if (n != want) return PyErr_Format(PyExc_TypeError, "%s: %zd arguments, expected %zd", kNames[id], n, want);
  if (!g_fn[id]) return PyErr_Format(PyExc_RuntimeError, "%s is not bound", kNames[id]);
  try {
    return PyLong_FromLong(f());
  } catch (const Bad&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

typedef PyObject* const* Args;

// (accumulated, q, k, probe_rows, probe_pos, sm_scale, lse_ext, scores, scores_per_head)
PyObject* probe(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kProbe, n, 9, [&]() -> int {
    const bool acc = PyObject_IsTrue(a[0]) != 0;
    const zc_tensor4 q = describe(a[1]), k = describe(a[2]);
    const auto* rows = ptr_as<const int32_t>(a[3]);
    const at::Tensor& pos = tensor_of(a[4]);
    const auto* posp = static_cast<const int32_t*>(pos.data_ptr());
    const int32_t P = (int32_t)pos.numel();
    const float scale = float_of(a[5]);
    const auto* lse = ptr_as<const float>(a[6]);
    auto* scores = ptr_as<float>(a[7]);
    auto* per_head = ptr_as<float>(a[8]);
    const hipStream_t st = current_stream();
    const Scratch ws = scratch(ZC_FN(kProbeWs, zc_probe_saliency_workspace)(q.B, q.H, k.L, P), tensor_of(a[1]), kScratchProbe, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(acc ? kAccumulated : kProbe, zc_probe_saliency);
    return unlocked(ws.use, [&] { return fn(&q, &k, rows, posp, P, scale, lse, scores, per_head, wp, wn, st); });
  });
}

// (q, k, v, sm_scale, out, lse, probe_pos, lse_probe)
PyObject* prefill(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPrefill, n, 8, [&]() -> int {
    const zc_tensor4 q = describe(a[0]), k = describe(a[1]), v = describe(a[2]), o = describe(a[4]);
    const float scale = float_of(a[3]);
    auto* lse = ptr_as<float>(a[5]);
    const int32_t P = a[6] == Py_None ? 0 : (int32_t)tensor_of(a[6]).numel();
    const auto* pos = P ? ptr_as<const int32_t>(a[6]) : nullptr;
    auto* lse_probe = P ? ptr_as<float>(a[7]) : nullptr;
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kPrefill, zc_prefill_attention);
    return unlocked([&] { return fn(&q, &k, &v, scale, &o, lse, pos, P, lse_probe, st); });
  });
}

// (scores, k, salient_idx, regular_idx, mask)
PyObject* select(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kSelect, n, 5, [&]() -> int {
    const at::Tensor& s = tensor_of(a[0]);
    if (s.dim() != 2) { PyErr_Format(PyExc_ValueError, "scores must be [B, L], got %d dimensions", (int)s.dim()); throw Bad(); }
    const int64_t B = s.size(0), L = s.size(1), k = int_of(a[1]);
    const auto* sp = static_cast<const float*>(s.data_ptr());
    auto *sal = ptr_as<int32_t>(a[2]), *reg = ptr_as<int32_t>(a[3]);
    auto* mask = ptr_as<uint8_t>(a[4]);
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kSelect, zc_select_salient);
    return unlocked([&] { return fn(sp, B, L, k, sal, reg, mask, nullptr, 0, st); });
  });
}

struct Lists { int64_t k, n_reg; const int32_t *sal, *reg; };
Lists lists_of(PyObject* sal, PyObject* reg) {
  Lists l;
  l.k = sal == Py_None ? 0 : tensor_of(sal).size(1);
  l.n_reg = reg == Py_None ? 0 : tensor_of(reg).size(1);
  l.sal = l.k ? ptr_as<const int32_t>(sal) : nullptr;
  l.reg = l.n_reg ? ptr_as<const int32_t>(reg) : nullptr;
  return l;
}

// (x, salient_idx, regular_idx, packed, pos_offset)
PyObject* quantize(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kQuantize, n, 5, [&]() -> int {
    const zc_tensor4 x = describe(a[0]);
    const Lists l = lists_of(a[1], a[2]);
    const Packed p(a[3]);
    const int64_t off = int_of(a[4]);
    const hipStream_t st = current_stream();
    const Scratch ws = scratch(ZC_FN(kQuantizeWs, zc_quantize_pack_workspace)(x.B, x.H, l.k + l.n_reg, x.D), tensor_of(a[0]),
                                kScratchQuantize, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kQuantize, zc_quantize_pack);
    return unlocked(ws.use, [&] { return fn(&x, l.sal, l.k, l.reg, l.n_reg, off, p.get(), wp, wn, st); });
  });
}

// (xk, xv, salient_idx, regular_idx, packedK, packedV, pos_offset)
PyObject* quantize_kv(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kQuantizeKV, n, 7, [&]() -> int {
    const zc_tensor4 xk = describe(a[0]), xv = describe(a[1]);
    const Lists l = lists_of(a[2], a[3]);
    const Packed pk(a[4]), pv(a[5]);
    const int64_t off = int_of(a[6]);
    const hipStream_t st = current_stream();
    const Scratch ws = scratch(ZC_FN(kQuantizeKVWs, zc_quantize_pack_kv_workspace)(xk.B, xk.H, l.k + l.n_reg, xk.D),
                                tensor_of(a[0]), kScratchQuantizeKV, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kQuantizeKV, zc_quantize_pack_kv);
    return unlocked(ws.use, [&] { return fn(&xk, &xv, l.sal, l.k, l.reg, l.n_reg, off, pk.get(), pv.get(), wp, wn, st); });
  });
}

// (use_static, q, packedK, packedV, tail_k, tail_v, tail_len, sm_scale, out, lse_out)
PyObject* decode(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kDecode, n, 10, [&]() -> int {
    const bool use_static = PyObject_IsTrue(a[0]) != 0;
    const zc_tensor4 q = describe(a[1], true);
    const Packed pk(a[2]), pv(a[3]);
    const int64_t T = int_of(a[6]);
    zc_tensor4 tk, tv;
    if (T) { tk = describe(a[4]); tv = describe(a[5]); }
    const zc_tensor4 *tkp = T ? &tk : nullptr, *tvp = T ? &tv : nullptr;
    const float scale = float_of(a[7]);
    void* out = tensor_of(a[8]).data_ptr();
    auto* lse = ptr_as<float>(a[9]);
    const hipStream_t st = current_stream();
    if (use_static) {
      const auto fn = ZC_FN(kDecodeStatic, zc_decode_attention_static);
      return unlocked(&g_static, [&] { return fn(&q, pk.get(), pv.get(), tkp, tvp, T, scale, out, lse, st); });
    }
    const Scratch ws = scratch(ZC_FN(kDecodeWs, zc_decode_attention_workspace)(q.B, q.H, q.D), tensor_of(a[1]), kScratchDecode, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kDecode, zc_decode_attention);
    return unlocked(ws.use, [&] { return fn(&q, pk.get(), pv.get(), tkp, tvp, T, scale, out, lse, wp, wn, st); });
  });
}

// (q, packedK, tail_k, tail_len, tail_pos0, lse, probs_out, sm_scale)
PyObject* probs(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kProbs, n, 8, [&]() -> int {
    const at::Tensor& out = tensor_of(a[6]);
    if (out.dim() != 3 || !out.is_contiguous() || out.scalar_type() != at::kFloat) {
      PyErr_SetString(PyExc_AssertionError, "probs_out must be a contiguous float32 [B, Hq, N] tensor");
      throw Bad();
    }
    const zc_tensor4 q = describe(a[0], true);
    const Packed pk(a[1]);
    const int64_t T = int_of(a[3]), pos0 = int_of(a[4]);
    zc_tensor4 tk;
    if (T) tk = describe(a[2]);
    const zc_tensor4* tkp = T ? &tk : nullptr;
    const auto* lse = static_cast<const float*>(tensor_of(a[5]).data_ptr());
    auto* po = static_cast<float*>(out.data_ptr());
    const int64_t N = out.size(2);
    const float scale = float_of(a[7]);
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kProbs, zc_decode_probs);
    return unlocked([&] { return fn(&q, pk.get(), tkp, T, pos0, scale, lse, po, N, st); });
  });
}

// (rows, row_len, n_out, normalize, scores)
PyObject* rows_saliency(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kRows, n, 5, [&]() -> int {
    const at::Tensor &rows = tensor_of(a[0]), &len = tensor_of(a[1]);
    if (rows.dim() != 4 || !rows.is_contiguous() || rows.scalar_type() != at::kFloat || len.scalar_type() != at::kInt) {
      PyErr_SetString(PyExc_AssertionError, "rows must be contiguous float32 [P, B, Hq, N], row_len int32");
      throw Bad();
    }
    const auto* rp = static_cast<const float*>(rows.data_ptr());
    const auto* lp = static_cast<const int32_t*>(len.data_ptr());
    const int32_t P = (int32_t)rows.size(0);
    const int64_t B = rows.size(1), H = rows.size(2), N = rows.size(3), n_out = int_of(a[2]);
    const int normalize = PyObject_IsTrue(a[3]) != 0;
    auto* sp = static_cast<float*>(tensor_of(a[4]).data_ptr());
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kRows, zc_rows_saliency);
    return unlocked([&] { return fn(rp, lp, P, B, H, N, n_out, normalize, sp, st); });
  });
}

// ---- the paged cache: what a call's tensors are is checked here (lengths and tables come from the caller's own bookkeeping) ----
[[noreturn]] void refuse(const char* what, const char* why) {
  PyErr_Format(PyExc_ValueError, "%s %s", what, why);
  throw Bad();
}
int g_device;                              // the current one, of the call that holds the interpreter lock (asked once a call)
void on_device(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) refuse(what, "must be on the GPU");
  if (g_device < 0) g_device = c10::hip::current_device();
  if (t.device().index() != g_device) refuse(what, "must be on the current device");
}
// int32, contiguous, of `n` elements (any number: -1); null for None.
int32_t* ints(PyObject* o, const char* what, int64_t n = -1) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor_of(o);
  on_device(t, what);
  if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse(what, "must be a contiguous int32 tensor");
  if (n >= 0 && t.numel() != n) refuse(what, "has another number of elements than the requests or rows ask for");
  return static_cast<int32_t*>(t.data_ptr());
}
// The capture that a stream is in.
struct Capture { bool on; unsigned long long id; };
Capture capture_of(hipStream_t stream) {
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  unsigned long long id = 0;
  if (hipStreamGetCaptureInfo(stream, &status, &id) != hipSuccess) {
    (void)hipGetLastError();
    return {false, 0};                     // (the default stream beside a capture)
  }
  return {status != hipStreamCaptureStatusNone, id};
}
// Whether torch's allocator has this memory in the pool of a graph.
bool of_a_graph(const at::Tensor& t) {
  const auto at = reinterpret_cast<uintptr_t>(t.data_ptr());
  try {
    for (const auto& s : c10::hip::HIPCachingAllocator::snapshot().segments)
      if (at >= (uintptr_t)s.address && at - (uintptr_t)s.address < s.total_size) return s.owner_private_pool_id != decltype(s.owner_private_pool_id){0, 0};
  } catch (const std::exception&) {
  }
  return false;                            // (an allocator that does not say)
}
// Scratch memory of a captured call: graphs share none, whatever stream they were captured on and whatever streams replay them.  In a
// capture that torch began it is the graph's, given back behind the call in the order of the capture.  In one that HIP alone
// knows of, what is given back would be anybody's while the graph is still replayed: it is kept, a buffer per capture and stream.
Scratch captured_scratch(size_t need, const at::Tensor& like, hipStream_t stream, unsigned long long id) {
  static bool of_torch = false;            // the capture `of`: asked once for each
  static unsigned long long of = 0;
  static auto* kept = new std::map<std::tuple<int, void*, unsigned long long>, at::Tensor>;
  const auto key = std::make_tuple((int)like.device().index(), (void*)stream, id);
  Scratch s;
  const auto have = kept->find(key);
  if (have != kept->end() && have->second.numel() >= (int64_t)need) {
    s.t = have->second;
  } else {
    s.t = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
    if (!of_torch || of != id) { of_torch = of_a_graph(s.t); of = id; }
    if (!of_torch) {
      if (have != kept->end()) g_captured->push_back(have->second);
      (*kept)[key] = s.t;
    }
  }
  s.ptr = s.t.data_ptr();
  s.bytes = s.t.numel();
  return s;
}
// Of a call over the pages: its graph's, or its stream's.
Scratch paged_scratch(size_t need, const at::Tensor& like, Kind kind, hipStream_t stream) {
  if (!need) return {};
  const Capture c = capture_of(stream);
  return c.on ? captured_scratch(need, like, stream, c.id) : scratch(need, like, kind, stream);
}
struct Table { int32_t* ptr; int64_t R, row, cols; };
Table table_of(PyObject* o, const char* what = "block_table") {
  const at::Tensor& t = tensor_of(o);
  on_device(t, what);
  if (t.scalar_type() != at::kInt || t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) refuse(what, "must be an int32 [R, max_blocks] tensor with rows that lie together");
  Table r = {static_cast<int32_t*>(t.data_ptr()), t.size(0), t.stride(0), t.size(1)};
  if (r.R < 2 || r.row < r.cols) {
    if (r.R > 1) refuse(what, "has rows that overlap");
    r.row = r.cols;
  }
  return r;
}
zc_tensor4 pool(PyObject* o, const char* what) {
  const zc_tensor4 r = describe(o);
  on_device(tensor_of(o), what);
  return r;
}
// Rows of a step's tokens: [T, H, D], or [1, H, T, D].
zc_tensor4 tokens(PyObject* o, const char* what) {
  const at::Tensor& t = tensor_of(o);
  zc_tensor4 r = describe(o, true);
  on_device(t, what);
  if (t.dim() == 3) {
    r.B = 1; r.H = t.size(1); r.L = t.size(0);
    r.sB = 0; r.sH = t.stride(1); r.sL = t.stride(0);
  }
  if (r.L <= 1) r.sL = r.D;                // (the stride of an axis of one element says nothing)
  if (r.H == 1) r.sH = 0;
  if (r.B == 1) r.sB = 0;
  return r;
}
int32_t int32_of(PyObject* o) {
  const int64_t v = int_of(o);
  return v > INT32_MAX ? INT32_MAX : v < INT32_MIN ? INT32_MIN : (int32_t)v;
}

// (q_len, kv_len, block_table, free_pages, n_free, page, T, q_start, slot_map, n_taken) -> (status, q_start, slot_map, n_taken); outputs
// that are None are allocated here: from Python the three allocations took longer than the kernel (8.0 -> 5.4 us a call).
PyObject* paged_tables(PyObject*, Args a, Py_ssize_t n) {
  at::Tensor made[3];
  PyObject* status = guarded(kPagedTables, n, 10, [&]() -> int {
    g_device = -1;
    const Table t = table_of(a[2]);
    const auto *q = ints(a[0], "q_len", t.R), *kv = ints(a[1], "kv_len", t.R);
    const at::Tensor& list = tensor_of(a[3]);
    const auto* free = ints(a[3], "free_pages");
    const auto* n_free = ints(a[4], "n_free", 1);
    const int64_t page = int_of(a[5]), T = int_of(a[6]), sizes[3] = {t.R + 1, T, 1};
    if (T < 0) refuse("T", "must not be negative");
    const char* const what[3] = {"q_start", "slot_map", "n_taken"};
    int32_t* out[3];
    // (one allocation for those that are missing, each from a multiple of 16 bytes on)
    at::Tensor memory;
    int64_t at = 0;
    for (int i = 0; i < 3; ++i) {
      if (a[7 + i] == Py_None) {
        if (!memory.defined()) memory = at::empty({(sizes[0] + 3) / 4 * 4 + (sizes[1] + 3) / 4 * 4 + sizes[2]}, list.options());
        made[i] = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(memory.storage()), memory.key_set(), memory.dtype());
        made[i].unsafeGetTensorImpl()->set_sizes_contiguous({sizes[i]});
        made[i].unsafeGetTensorImpl()->set_storage_offset(at);
        out[i] = static_cast<int32_t*>(made[i].data_ptr());
        at += (sizes[i] + 3) / 4 * 4;
      } else {
        made[i] = tensor_of(a[7 + i]);
        out[i] = ints(a[7 + i], what[i], sizes[i]);
      }
    }
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kPagedTables, zc_paged_tables);
    return unlocked([&] { return fn(q, kv, t.R, t.ptr, t.row, t.cols, free, list.numel(), n_free, page, out[0], out[1], T, out[2], st); });
  });
  if (!status) return nullptr;
  PyObject* all = PyTuple_New(4);
  if (!all) { Py_DECREF(status); return nullptr; }
  PyTuple_SET_ITEM(all, 0, status);
  for (int i = 0; i < 3; ++i) {
    PyObject* o = THPVariable_Wrap(made[i]);
    if (!o) { Py_DECREF(all); return nullptr; }
    PyTuple_SET_ITEM(all, 1 + i, o);
  }
  return all;
}

// (k, v, slot_map, k_pages, v_pages)
PyObject* paged_store(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedStore, n, 5, [&]() -> int {
    g_device = -1;
    const zc_tensor4 k = tokens(a[0], "k"), v = tokens(a[1], "v"), kp = pool(a[3], "k_pages"), vp = pool(a[4], "v_pages");
    const auto* slots = ints(a[2], "slot_map", k.L);
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kPagedStore, zc_paged_store);
    return unlocked([&] { return fn(&k, &v, slots, &kp, &vp, st); });
  });
}

// (k_pages, v_pages, block_table, kv_len, k_out, v_out)
PyObject* paged_load(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedLoad, n, 6, [&]() -> int {
    g_device = -1;
    const zc_tensor4 kp = pool(a[0], "k_pages"), vp = pool(a[1], "v_pages"), k = pool(a[4], "k_out"), v = pool(a[5], "v_out");
    const Table t = table_of(a[2]);
    const auto* kv = ints(a[3], "kv_len", t.R);
    if (k.B != t.R || v.B != t.R) refuse("k_out and v_out", "must have a batch element for each row of block_table");
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kPagedLoad, zc_paged_load);
    return unlocked([&] { return fn(&kp, &vp, t.ptr, t.row, t.cols, kv, &k, &v, st); });
  });
}

// (q, k_pages, v_pages, block_table, q_start, kv_len, window, sinks, sm_scale, out, lse)
PyObject* paged_attention(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedAttention, n, 11, [&]() -> int {
    g_device = -1;
    const zc_tensor4 q = tokens(a[0], "q"), kp = pool(a[1], "k_pages"), vp = pool(a[2], "v_pages"), o = tokens(a[9], "out");
    const Table t = table_of(a[3]);
    const auto *start = ints(a[4], "q_start", t.R + 1), *kv = ints(a[5], "kv_len", t.R);
    const int32_t window = int32_of(a[6]), sinks = int32_of(a[7]);
    const float scale = float_of(a[8]);
    float* lse = nullptr;
    if (a[10] != Py_None) {
      const at::Tensor& l = tensor_of(a[10]);
      on_device(l, "lse");
      if (l.scalar_type() != at::kFloat || !l.is_contiguous() || l.numel() != q.H * q.L) refuse("lse", "must be a contiguous float32 [Hq, T] tensor");
      lse = static_cast<float*>(l.data_ptr());
    }
    const hipStream_t st = current_stream();
    const size_t need = ZC_FN(kPagedAttentionWs, zc_paged_attention_workspace)(t.R, q.L, q.H, kp.H, q.D);
    const Scratch ws = paged_scratch(need, tensor_of(a[0]), kScratchPaged, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kPagedAttention, zc_paged_attention);
    return unlocked(ws.use, [&] { return fn(&q, &kp, &vp, t.ptr, t.row, t.cols, start, kv, t.R, window, sinks, scale, &o, lse, wp, wn, st); });
  });
}

// (q, k_pages, v_pages, prefix_table, prefix_len, group_start, block_table, q_start, kv_len, sm_scale, out, lse)
PyObject* paged_shared(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedShared, n, 12, [&]() -> int {
    g_device = -1;
    const zc_tensor4 q = tokens(a[0], "q"), kp = pool(a[1], "k_pages"), vp = pool(a[2], "v_pages"), o = tokens(a[10], "out");
    const Table pre = table_of(a[3], "prefix_table"), t = table_of(a[6]);
    const auto *len = ints(a[4], "prefix_len", pre.R), *groups = ints(a[5], "group_start", pre.R + 1);
    const auto *start = ints(a[7], "q_start", t.R + 1), *kv = ints(a[8], "kv_len", t.R);
    const float scale = float_of(a[9]);
    float* lse = nullptr;
    if (a[11] != Py_None) {
      const at::Tensor& l = tensor_of(a[11]);
      on_device(l, "lse");
      if (l.scalar_type() != at::kFloat || !l.is_contiguous() || l.numel() != q.H * q.L) refuse("lse", "must be a contiguous float32 [Hq, T] tensor");
      lse = static_cast<float*>(l.data_ptr());
    }
    const hipStream_t st = current_stream();
    const size_t need = ZC_FN(kPagedSharedWs, zc_paged_shared_attention_workspace)(pre.R, t.R, q.L, q.H, kp.H, q.D);
    const Scratch ws = paged_scratch(need, tensor_of(a[0]), kScratchShared, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kPagedShared, zc_paged_shared_attention);
    return unlocked(ws.use, [&] {
      return fn(&q, &kp, &vp, pre.ptr, pre.row, pre.cols, len, groups, pre.R, t.ptr, t.row, t.cols, start, kv, t.R, scale, &o, lse, wp, wn, st);
    });
  });
}

// Gathered weights beside the pages: float32 [N, Hkv, page].
float* scores_of(PyObject* o, const zc_tensor4& pages) {
  const at::Tensor& t = tensor_of(o);
  on_device(t, "scores");
  if (t.scalar_type() != at::kFloat || !t.is_contiguous() || t.dim() != 3 || t.size(0) != pages.B || t.size(1) != pages.H || t.size(2) != pages.L)
    refuse("scores", "must be a contiguous float32 [N, Hkv, page] tensor");
  return static_cast<float*>(t.data_ptr());
}

// (q, k_pages, block_table, q_start, kv_len, lse, scores, window, sinks, sm_scale, decay)
PyObject* paged_scores(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedScores, n, 11, [&]() -> int {
    g_device = -1;
    const zc_tensor4 q = tokens(a[0], "q"), kp = pool(a[1], "k_pages");
    const Table t = table_of(a[2]);
    const auto *start = ints(a[3], "q_start", t.R + 1), *kv = ints(a[4], "kv_len", t.R);
    const at::Tensor& l = tensor_of(a[5]);
    on_device(l, "lse");
    if (l.scalar_type() != at::kFloat || !l.is_contiguous() || l.numel() != q.H * q.L) refuse("lse", "must be a contiguous float32 [Hq, T] tensor");
    const auto* lse = static_cast<const float*>(l.data_ptr());
    float* scores = scores_of(a[6], kp);
    const int32_t window = int32_of(a[7]), sinks = int32_of(a[8]);
    const float scale = float_of(a[9]), decay = float_of(a[10]);
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kPagedScores, zc_paged_scores);
    return unlocked([&] { return fn(&q, &kp, t.ptr, t.row, t.cols, start, kv, t.R, window, sinks, scale, lse, decay, scores, st); });
  });
}

// (k_pages, v_pages, scores, block_table, kv_len, keep, most, sinks, recent, together, new_len, kept, free_pages, n_free, n_freed)
PyObject* paged_evict(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kPagedEvict, n, 15, [&]() -> int {
    g_device = -1;
    const zc_tensor4 kp = pool(a[0], "k_pages"), vp = pool(a[1], "v_pages");
    float* scores = scores_of(a[2], kp);
    const Table t = table_of(a[3]);
    const auto *kv = ints(a[4], "kv_len", t.R), *keep = ints(a[5], "keep", t.R);
    const int64_t most = int_of(a[6]);
    const int32_t sinks = int32_of(a[7]), recent = int32_of(a[8]);
    const int together = PyObject_IsTrue(a[9]);
    if (together < 0) throw Bad();
    if (most < 0) refuse("most", "must not be negative");
    auto *len = ints(a[10], "new_len", t.R), *kept = ints(a[11], "kept", t.R * (together ? 1 : kp.H) * most);
    int32_t* free = ints(a[12], "free_pages");
    const int64_t list = free ? tensor_of(a[12]).numel() : 0;
    const auto* n_free = ints(a[13], "n_free", 1);
    auto* n_freed = ints(a[14], "n_freed", 1);
    const hipStream_t st = current_stream();
    const size_t need = ZC_FN(kPagedEvictWs, zc_paged_evict_workspace)(t.R, kp.H, t.cols, kp.L, together);
    const Scratch ws = paged_scratch(need, tensor_of(a[0]), kScratchEvict, st);
    void* wp = ws.ptr;
    const size_t wn = ws.bytes;
    const auto fn = ZC_FN(kPagedEvict, zc_paged_evict);
    return unlocked(ws.use, [&] {
      return fn(&kp, &vp, scores, t.ptr, t.row, t.cols, kv, keep, t.R, most, sinks, recent, together, len, kept, free, list, n_free, n_freed, wp, wn, st);
    });
  });
}

// (packed, out)
PyObject* dequantize(PyObject*, Args a, Py_ssize_t n) {
  return guarded(kDequantize, n, 2, [&]() -> int {
    const Packed p(a[0]);
    const zc_tensor4 o = describe(a[1]);
    const hipStream_t st = current_stream();
    const auto fn = ZC_FN(kDequantize, zc_dequantize_cache);
    return unlocked([&] { return fn(p.get(), &o, st); });
  });
}

// names(): the entry points bind() wants; bind(addresses): their addresses, in that order
PyObject* names(PyObject*, PyObject*) {
  PyObject* t = PyTuple_New(kFnCount);
  for (int i = 0; t && i < kFnCount; ++i) PyTuple_SET_ITEM(t, i, PyUnicode_FromString(kNames[i]));
  return t;
}
PyObject* bind(PyObject*, PyObject* seq) {
  if (!PyTuple_Check(seq) || PyTuple_GET_SIZE(seq) != kFnCount) return PyErr_Format(PyExc_TypeError, "bind: a tuple of %d addresses", (int)kFnCount);
  void* got[kFnCount];
  for (int i = 0; i < kFnCount; ++i) {
    got[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(seq, i));
    if (!got[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "bind: %s has no address", kNames[i]);
  }
  for (int i = 0; i < kFnCount; ++i) g_fn[i] = got[i];
  Py_RETURN_NONE;
}

#define ZC_METHOD(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    {"names", names, METH_NOARGS, nullptr},
    {"bind", bind, METH_O, nullptr},
    ZC_METHOD("probe", probe),
    ZC_METHOD("prefill", prefill),
    ZC_METHOD("select", select),
    ZC_METHOD("quantize", quantize),
    ZC_METHOD("quantize_kv", quantize_kv),
    ZC_METHOD("decode", decode),
    ZC_METHOD("probs", probs),
    ZC_METHOD("rows_saliency", rows_saliency),
    ZC_METHOD("dequantize", dequantize),
    ZC_METHOD("paged_tables", paged_tables),
    ZC_METHOD("paged_store", paged_store),
    ZC_METHOD("paged_load", paged_load),
    ZC_METHOD("paged_attention", paged_attention),
    ZC_METHOD("paged_shared", paged_shared),
    ZC_METHOD("paged_scores", paged_scores),
    ZC_METHOD("paged_evict", paged_evict),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_zc_host", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__zc_host() {
  g_scratch = new std::map<std::tuple<int, int, void*>, Scratch>();   // (neither is freed: tensors must not outlive the allocator at exit)
  g_captured = new std::vector<at::Tensor>();
  return PyModule_Create(&kModule);
}
