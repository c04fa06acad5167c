// The Python side of the calls that take microseconds (draft sampling, verification, one projection, the operators of a
// caller's own drafter): argument checks, output tensors and the call into the C ABI in one native function each.
//
// What it is for: on the host such a call used to take longer than its kernels on the GPU.  Two torch.empty() of a few bytes
// 4.3 us, attribute look-ups 2, ctypes 1.2, the launches 2.1 each: a verification of one sequence 12.4 us, a draw 7.2, a small projection
// 9.1; this way 7.1, 4.5 and 4.4.  No arithmetic of the method is here.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <vector>

#include "../../include/hsd.h"

namespace {

decltype(&hsd_draft_sample) draft_sample_fn = nullptr;
decltype(&hsd_verify_workspace_bytes) verify_bytes_fn = nullptr;
decltype(&hsd_verify_level) verify_level_fn = nullptr;
decltype(&hsd_gemm_workspace_bytes) gemm_bytes_fn = nullptr;
decltype(&hsd_gemm_bf16) gemm_fn = nullptr;
decltype(&hsd_gemm_status) gemm_status_fn = nullptr;
decltype(&hsd_strerror) strerror_fn = nullptr;
decltype(&hsd_kv_append) kv_append_fn = nullptr, kv_append_zeros_fn = nullptr;
decltype(&hsd_paged_attention_workspace_bytes) attention_bytes_fn = nullptr;
decltype(&hsd_paged_attention) attention_fn = nullptr;
decltype(&hsd_gemm_w4_workspace_bytes) gemm_w4_bytes_fn = nullptr;
decltype(&hsd_gemm_w4) gemm_w4_fn = nullptr;
decltype(&hsd_token_logprobs) logprobs_fn = nullptr;
decltype(&hsd_kv_append_norm) kv_append_norm_fn = nullptr;
decltype(&hsd_quantize_rows) quantize_fn = nullptr;
decltype(&hsd_gemm_w8_workspace_bytes) gemm_w8_bytes_fn = nullptr;
decltype(&hsd_gemm_w8) gemm_w8_fn = nullptr;
decltype(&hsd_prefix_attention_workspace_bytes) prefix_bytes_fn = nullptr;
decltype(&hsd_prefix_attention) prefix_fn = nullptr;
PyObject *error_class = nullptr;

struct Failed {};                                          // a Python exception is set

const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor, got %.80s", Py_TYPE(o)->tp_name);
    throw Failed();
  }
  return THPVariable_Unpack(o);
}
void *device_data(const at::Tensor &t) {
  if (!t.is_cuda() || !t.is_contiguous()) {
    PyErr_SetString(error_class, "expected a contiguous CUDA tensor");
    throw Failed();
  }
  return t.data_ptr();
}
const at::Tensor &shaped(PyObject *o, int64_t dims) {
  const at::Tensor &t = tensor(o);
  if (t.dim() != dims) {
    PyErr_Format(PyExc_ValueError, "expected %d dimensions, got %d", (int)dims, (int)t.dim());
    throw Failed();
  }
  return t;
}
int dtype_code(const at::Tensor &t) {
  if (t.scalar_type() == at::kFloat) return HSD_F32;
  if (t.scalar_type() == at::kBFloat16) return HSD_BF16;
  PyErr_Format(error_class, "unsupported logits dtype %s", c10::toString(t.scalar_type()));
  throw Failed();
}
uint64_t word(PyObject *o) {                               // modulo 2^64, as a C prototype takes a Python integer
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Failed();
  return v;
}
void check(int status) {
  if (!status) return;
  PyErr_Format(error_class, "hsd call failed: %s (%d)", strerror_fn(status), status);
  throw Failed();
}
void arguments(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
  throw Failed();
}
template <class F> int released(F &&f) {                   // other threads run while the call is made, as with ctypes
  PyThreadState *state = PyEval_SaveThread();
  const int status = f();
  PyEval_RestoreThread(state);
  return status;
}
void *current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// init(addresses of the C functions, in the order below; error class)
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 21);
    draft_sample_fn = reinterpret_cast<decltype(draft_sample_fn)>(word(args[0]));
    verify_bytes_fn = reinterpret_cast<decltype(verify_bytes_fn)>(word(args[1]));
    verify_level_fn = reinterpret_cast<decltype(verify_level_fn)>(word(args[2]));
    gemm_bytes_fn = reinterpret_cast<decltype(gemm_bytes_fn)>(word(args[3]));
    gemm_fn = reinterpret_cast<decltype(gemm_fn)>(word(args[4]));
    gemm_status_fn = reinterpret_cast<decltype(gemm_status_fn)>(word(args[5]));
    strerror_fn = reinterpret_cast<decltype(strerror_fn)>(word(args[6]));
    kv_append_fn = reinterpret_cast<decltype(kv_append_fn)>(word(args[7]));
    attention_bytes_fn = reinterpret_cast<decltype(attention_bytes_fn)>(word(args[8]));
    attention_fn = reinterpret_cast<decltype(attention_fn)>(word(args[9]));
    gemm_w4_bytes_fn = reinterpret_cast<decltype(gemm_w4_bytes_fn)>(word(args[10]));
    gemm_w4_fn = reinterpret_cast<decltype(gemm_w4_fn)>(word(args[11]));
    logprobs_fn = reinterpret_cast<decltype(logprobs_fn)>(word(args[12]));
    kv_append_zeros_fn = reinterpret_cast<decltype(kv_append_zeros_fn)>(word(args[13]));
    kv_append_norm_fn = reinterpret_cast<decltype(kv_append_norm_fn)>(word(args[14]));
    quantize_fn = reinterpret_cast<decltype(quantize_fn)>(word(args[15]));
    gemm_w8_bytes_fn = reinterpret_cast<decltype(gemm_w8_bytes_fn)>(word(args[16]));
    gemm_w8_fn = reinterpret_cast<decltype(gemm_w8_fn)>(word(args[17]));
    prefix_bytes_fn = reinterpret_cast<decltype(prefix_bytes_fn)>(word(args[18]));
    prefix_fn = reinterpret_cast<decltype(prefix_fn)>(word(args[19]));
    Py_INCREF(args[20]);
    error_class = args[20];
    Py_RETURN_NONE;
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// draft_sample(logits [batch, rows, vocab], seed, call_serial, out_tokens or None)
PyObject *draft_sample(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 4);
    const at::Tensor &logits = shaped(args[0], 3);
    void *data = device_data(logits);
    const int dtype = dtype_code(logits);
    const int batch = (int)logits.size(0), rows = (int)logits.size(1), vocab = (int)logits.size(2);
    const uint64_t seed = word(args[1]), serial = word(args[2]);
    at::Tensor out = args[3] == Py_None ? at::empty({batch, rows}, logits.options().dtype(at::kInt).requires_grad(false)) : tensor(args[3]);
    int32_t *to = static_cast<int32_t *>(device_data(out));
    void *stream = current_stream();
    check(released([&] { return draft_sample_fn(data, batch, rows, vocab, dtype, seed, serial, stream, to); }));
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// verify_level(level, target [batch, t + 1, vocab], draft [batch, t, vocab], tokens [batch, t], seed, call_serial, workspace, out_tokens,
// out_n_accepted), the last three or None
PyObject *verify_level(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 9);
    const int level = (int)word(args[0]);
    const at::Tensor &target = shaped(args[1], 3);
    void *p = device_data(target);
    const int batch = (int)target.size(0), t = (int)target.size(1) - 1, vocab = (int)target.size(2);
    void *q = t > 0 ? device_data(tensor(args[2])) : nullptr;
    int32_t *tokens = t > 0 ? static_cast<int32_t *>(device_data(tensor(args[3]))) : nullptr;
    const int dtype = dtype_code(target);
    const uint64_t seed = word(args[4]), serial = word(args[5]);
    const auto options = target.options().requires_grad(false);
    at::Tensor ws = args[6] == Py_None ? at::empty({std::max<int64_t>(16, (int64_t)verify_bytes_fn(batch, t))}, options.dtype(at::kByte)) : tensor(args[6]);
    at::Tensor out = args[7] == Py_None ? at::empty({batch, t + 1}, options.dtype(at::kInt)) : tensor(args[7]);
    at::Tensor accepted = args[8] == Py_None ? at::empty({batch}, options.dtype(at::kInt)) : tensor(args[8]);
    void *scratch = device_data(ws), *to = device_data(out), *count = device_data(accepted), *stream = current_stream();
    check(released([&] {
      return verify_level_fn(level, p, q, tokens, batch, t, vocab, dtype, seed, serial, scratch, (size_t)ws.numel(), stream,
                             static_cast<int32_t *>(to), static_cast<int32_t *>(count));
    }));
    PyObject *first = THPVariable_Wrap(std::move(out)), *second = THPVariable_Wrap(std::move(accepted)), *both = nullptr;
    if (first && second) both = PyTuple_Pack(2, first, second);
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// If the caller asks for it: the stream is waited for, a device-side wait that gave up is an error.
void check_waits(PyObject *wanted, void *workspace, void *stream) {
  const int yes = PyObject_IsTrue(wanted);
  if (yes < 0) throw Failed();
  if (yes) check(released([&] { return gemm_status_fn(workspace, stream); }));
}

// gemm_bf16(A [R, K], W [N, K], out or None, workspace or None, check)
PyObject *gemm_bf16(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 5);
    const at::Tensor &a = shaped(args[0], 2), &w = tensor(args[1]);
    const int R = (int)a.size(0), K = (int)a.size(1), N = (int)w.size(0);
    const size_t need = gemm_bytes_fn(R, N, K);
    if (need == 0) {
      PyErr_Format(error_class, "hsd_gemm_bf16: unsupported shape R=%d N=%d K=%d", R, N, K);
      throw Failed();
    }
    void *pa = device_data(a), *pw = device_data(w);
    const auto options = a.options().requires_grad(false);
    at::Tensor ws = args[3] == Py_None ? at::empty({(int64_t)need + 256}, options.dtype(at::kByte)) : tensor(args[3]);
    at::Tensor out = args[2] == Py_None ? at::empty({R, N}, options.dtype(at::kFloat)) : tensor(args[2]);
    float *to = static_cast<float *>(device_data(out));
    const uintptr_t start = reinterpret_cast<uintptr_t>(ws.data_ptr()), base = (start + 255) / 256 * 256;
    void *scratch = reinterpret_cast<void *>(base), *stream = current_stream();
    const int64_t left = ws.numel() - (int64_t)(base - start);
    check(released([&] { return gemm_fn(pa, R, K, pw, N, to, scratch, left < 0 ? 0 : (size_t)left, stream); }));
    check_waits(args[4], scratch, stream);
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// The operators below launch on their tensors' device, whichever is current, on that device's current stream.
[[noreturn]] void refuse(const char *what) {
  PyErr_SetString(error_class, what);
  throw Failed();
}
// A tensor of this type on the device of `like` (any CUDA device without one).
const at::Tensor &typed(PyObject *o, const char *name, at::ScalarType type, const at::Tensor *like = nullptr) {
  const at::Tensor &t = tensor(o);
  if (!t.is_cuda()) refuse("expected a CUDA tensor");
  if (t.scalar_type() != type) {
    PyErr_Format(error_class, "%s: expected %s, got %s", name, c10::toString(type), c10::toString(t.scalar_type()));
    throw Failed();
  }
  if (like && t.device() != like->device()) {
    PyErr_Format(error_class, "%s is on another device", name);
    throw Failed();
  }
  return t;
}
const at::Tensor &sized(const at::Tensor &t, const char *name, at::IntArrayRef sizes) {
  if (!t.is_contiguous()) refuse("expected a contiguous CUDA tensor");
  if (t.sizes() != sizes) {
    PyErr_Format(PyExc_ValueError, "%s has another shape than the call's other tensors ask for", name);
    throw Failed();
  }
  return t;
}
const at::Tensor &dims(const at::Tensor &t, const char *name, int64_t n) {
  if (t.dim() != n) {
    PyErr_Format(PyExc_ValueError, "%s: expected %d dimensions, got %d", name, (int)n, (int)t.dim());
    throw Failed();
  }
  return t;
}
int count(int64_t n) {
  if (n > INT32_MAX) refuse("a size is over 2^31 - 1");
  return (int)n;
}
// An output on the current device.  (at::empty without its way through the dispatcher: five of them took longer on the host, 4 us, than a
// short call's kernel.)
at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type) {
  return at::detail::empty_generic(sizes, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
}
at::ScalarType cache_type(const at::Tensor &t, const char *name) {
  if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) {
    PyErr_Format(error_class, "%s: unsupported dtype %s", name, c10::toString(t.scalar_type()));
    throw Failed();
  }
  return t.scalar_type();
}
// Pools [n_kv_heads, n_pages, page_size, head_dim], in any order in memory with head_dim innermost.
hsd_kv_pool pools(PyObject *ko, PyObject *vo, const at::Tensor *like) {
  const at::Tensor &k = dims(tensor(ko), "k_pool", 4), &v = tensor(vo);
  const at::ScalarType type = cache_type(k, "k_pool");
  typed(ko, "k_pool", type, like);
  typed(vo, "v_pool", type, &k);
  if (k.sizes() != v.sizes() || k.strides() != v.strides()) {
    PyErr_SetString(PyExc_ValueError, "k_pool and v_pool differ in their sizes or strides");
    throw Failed();
  }
  if (k.stride(3) != 1 && k.size(3) != 1) refuse("the pools' last dimension has to be contiguous");
  return {k.data_ptr(), v.data_ptr(), type == at::kFloat ? HSD_F32 : HSD_BF16, count(k.size(1)), count(k.size(2)), k.stride(0), k.stride(1), k.stride(2)};
}

// What both appends take; gains null: without a norm.
struct Gains { PyObject *q, *k, *eps; };
PyObject *append(PyObject *qkv_o, PyObject *k_o, PyObject *v_o, PyObject *table_o, PyObject *lens_o, PyObject *rope_o, PyObject *starts_o, PyObject *out_o, const Gains *gains) {
  const at::Tensor &qkv = dims(tensor(qkv_o), "qkv", 3);
  const at::ScalarType source = cache_type(qkv, "qkv");
  typed(qkv_o, "qkv", source);
  const hsd_kv_pool pool = pools(k_o, v_o, &qkv);
  const int64_t nkv = tensor(k_o).size(0), hd = qkv.size(2), nq = qkv.size(1) - 2 * nkv;
  if (nq < 0 || hd != tensor(k_o).size(3)) {
    PyErr_SetString(PyExc_ValueError, "qkv has fewer heads than twice the pools' or another head size");
    throw Failed();
  }
  if ((hd > 1 && qkv.stride(2) != 1) || (qkv.size(1) > 1 && qkv.stride(1) != hd)) refuse("qkv: the heads of a row have to be contiguous");
  const at::Tensor &table = dims(typed(table_o, "page_table", at::kInt, &qkv), "page_table", 2);
  const int64_t batch = table.size(0), rows = qkv.size(0);
  sized(table, "page_table", {batch, table.size(1)});
  const at::Tensor &lens = sized(typed(lens_o, "kv_lens", at::kInt, &qkv), "kv_lens", {batch});
  const at::Tensor &rope = dims(typed(rope_o, "rope", at::kFloat, &qkv), "rope", 3);
  sized(rope, "rope", {rope.size(0), 2, hd / 2});
  const int32_t *starts = nullptr;
  if (starts_o != Py_None) starts = static_cast<const int32_t *>(sized(typed(starts_o, "row_starts", at::kInt, &qkv), "row_starts", {batch + 1}).data_ptr());
  const at::ScalarType type = pool.dtype == HSD_F32 ? at::kFloat : at::kBFloat16;
  const void *gain[2] = {nullptr, nullptr};
  at::ScalarType gain_type = at::kFloat;
  double eps = 0.;
  if (gains) {
    const char *names[2] = {"q_gain", "k_gain"};
    PyObject *given[2] = {gains->q, gains->k};
    if (given[0] != Py_None) gain_type = cache_type(tensor(given[0]), names[0]);
    else if (given[1] != Py_None) gain_type = cache_type(tensor(given[1]), names[1]);
    for (int x = 0; x < 2; ++x)
      if (given[x] != Py_None) gain[x] = sized(typed(given[x], names[x], gain_type, &qkv), names[x], {hd}).data_ptr();
    eps = PyFloat_AsDouble(gains->eps);
    if (eps == -1. && PyErr_Occurred()) throw Failed();
  }
  const c10::cuda::CUDAGuard guard(qkv.device());
  at::Tensor out = out_o == Py_None ? fresh({rows, nq, hd}, type) : sized(typed(out_o, "q_out", type, &qkv), "q_out", {rows, nq, hd});
  void *from = qkv.data_ptr(), *to = out.data_ptr(), *stream = current_stream();
  const int n_rows = count(rows), heads = count(nq), kv_heads = count(nkv), dim = count(hd), n_batch = count(batch), pages = count(table.size(1)), positions = count(rope.size(0));
  const long long stride = rows > 1 ? qkv.stride(0) : qkv.size(1) * hd;
  const int dtype = source == at::kFloat ? HSD_F32 : HSD_BF16;
  const int32_t *n_lens = static_cast<const int32_t *>(lens.data_ptr()), *n_table = static_cast<const int32_t *>(table.data_ptr());
  const float *angles = static_cast<const float *>(rope.data_ptr());
  const auto call = out_o == Py_None ? kv_append_zeros_fn : kv_append_fn;                  // (fresh memory holds anything)
  check(released([&] {
    if (gains) return kv_append_norm_fn(from, dtype, n_rows, stride, heads, kv_heads, dim, gain[0], gain[1], gain_type == at::kFloat ? HSD_F32 : HSD_BF16, (float)eps,
                                        starts, n_lens, n_batch, n_table, pages, angles, positions, &pool, out_o == Py_None, to, stream);
    return call(from, dtype, n_rows, stride, heads, kv_heads, dim, starts, n_lens, n_batch, n_table, pages, angles, positions, &pool, to, stream);
  }));
  return THPVariable_Wrap(std::move(out));
}

// kv_append(qkv [rows, nq + 2 nkv, hd], k_pool, v_pool, page_table [batch, pages], kv_lens [batch], rope [positions, 2, hd / 2],
// row_starts [batch + 1] or None, q_out or None)
PyObject *kv_append(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 8);
    return append(args[0], args[1], args[2], args[3], args[4], args[5], args[6], args[7], nullptr);
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// kv_append_norm(qkv, q_gain [hd] or None, k_gain [hd] or None, eps, then as kv_append)
PyObject *kv_append_norm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 11);
    const Gains gains = {args[1], args[2], args[3]};
    return append(args[0], args[4], args[5], args[6], args[7], args[8], args[9], args[10], &gains);
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// paged_attention(q [batch, nq, hd], k_pool, v_pool, page_table [batch, pages], kv_lens [batch], scale or None, workspace or None, out or None)
PyObject *paged_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 8);
    const at::Tensor &q = dims(tensor(args[0]), "q", 3);
    const hsd_kv_pool pool = pools(args[1], args[2], &q);
    const at::Tensor &k = tensor(args[1]);
    const int64_t batch = q.size(0), nq = q.size(1), hd = q.size(2);
    sized(typed(args[0], "q", k.scalar_type(), &k), "q", {batch, nq, k.size(3)});
    const at::Tensor &table = dims(typed(args[3], "page_table", at::kInt, &q), "page_table", 2);
    sized(table, "page_table", {batch, table.size(1)});
    const at::Tensor &lens = sized(typed(args[4], "kv_lens", at::kInt, &q), "kv_lens", {batch});
    double scale = 1. / std::sqrt((double)hd);
    if (args[5] != Py_None) {
      scale = PyFloat_AsDouble(args[5]);
      if (scale == -1. && PyErr_Occurred()) throw Failed();
    }
    const int n_batch = count(batch), heads = count(nq), kv_heads = count(k.size(0)), dim = count(hd), pages = count(table.size(1));
    const size_t need = attention_bytes_fn(heads, kv_heads, dim);
    if (need == 0) {
      PyErr_Format(error_class, "hsd_paged_attention: unsupported heads: %d queries, %d keys of %d", heads, kv_heads, dim);
      throw Failed();
    }
    const c10::cuda::CUDAGuard guard(q.device());
    at::Tensor ws = args[6] == Py_None ? fresh({(int64_t)need}, at::kByte) : typed(args[6], "workspace", at::kByte, &q);
    if (!ws.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    at::Tensor out = args[7] == Py_None ? fresh({batch, nq, hd}, q.scalar_type()) : sized(typed(args[7], "out", q.scalar_type(), &q), "out", {batch, nq, hd});
    void *from = q.data_ptr(), *to = out.data_ptr(), *scratch = ws.data_ptr(), *stream = current_stream();
    check(released([&] {
      return attention_fn(from, n_batch, heads, kv_heads, dim, &pool, static_cast<const int32_t *>(table.data_ptr()), pages,
                          static_cast<const int32_t *>(lens.data_ptr()), (float)scale, scratch, (size_t)ws.numel(), to, stream);
    }));
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// prefix_attention(q [rows, nq, hd], k_pool, v_pool, page_table [batch, pages], kv_lens [batch], prefix_pages [n], prefix_len [1],
// row_starts [batch + 1] or None, scale or None, workspace or None, out or None, check)
PyObject *prefix_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 12);
    const at::Tensor &q = dims(tensor(args[0]), "q", 3);
    const hsd_kv_pool pool = pools(args[1], args[2], &q);
    const at::Tensor &k = tensor(args[1]);
    const int64_t rows = q.size(0), nq = q.size(1), hd = q.size(2);
    sized(typed(args[0], "q", k.scalar_type(), &k), "q", {rows, nq, k.size(3)});
    const at::Tensor &table = dims(typed(args[3], "page_table", at::kInt, &q), "page_table", 2);
    const int64_t batch = table.size(0);
    sized(table, "page_table", {batch, table.size(1)});
    const at::Tensor &lens = sized(typed(args[4], "kv_lens", at::kInt, &q), "kv_lens", {batch});
    const at::Tensor &prefix = dims(typed(args[5], "prefix_pages", at::kInt, &q), "prefix_pages", 1);
    sized(prefix, "prefix_pages", {prefix.size(0)});
    const at::Tensor &length = sized(typed(args[6], "prefix_len", at::kInt, &q), "prefix_len", {1});
    const int32_t *starts = nullptr;
    if (args[7] != Py_None) starts = static_cast<const int32_t *>(sized(typed(args[7], "row_starts", at::kInt, &q), "row_starts", {batch + 1}).data_ptr());
    double scale = 1. / std::sqrt((double)hd);
    if (args[8] != Py_None) {
      scale = PyFloat_AsDouble(args[8]);
      if (scale == -1. && PyErr_Occurred()) throw Failed();
    }
    const int n_rows = count(rows), heads = count(nq), kv_heads = count(k.size(0)), dim = count(hd), n_batch = count(batch), pages = count(table.size(1)), front = count(prefix.size(0));
    const size_t need = prefix_bytes_fn(n_rows, heads, kv_heads, dim);
    if (need == 0) {
      PyErr_Format(error_class, "hsd_prefix_attention: unsupported sizes: %d rows, %d queries, %d keys of %d", n_rows, heads, kv_heads, dim);
      throw Failed();
    }
    const c10::cuda::CUDAGuard guard(q.device());
    at::Tensor ws = args[9] == Py_None ? fresh({(int64_t)need}, at::kByte) : typed(args[9], "workspace", at::kByte, &q);
    if (!ws.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    at::Tensor out = args[10] == Py_None ? fresh({rows, nq, hd}, q.scalar_type()) : sized(typed(args[10], "out", q.scalar_type(), &q), "out", {rows, nq, hd});
    void *from = q.data_ptr(), *to = out.data_ptr(), *scratch = ws.data_ptr(), *stream = current_stream();
    const bool own = args[10] == Py_None;                                                  // (fresh memory holds anything)
    check(released([&] {
      return prefix_fn(from, n_rows, heads, kv_heads, dim, &pool, static_cast<const int32_t *>(table.data_ptr()), pages, static_cast<const int32_t *>(lens.data_ptr()), starts,
                       n_batch, static_cast<const int32_t *>(prefix.data_ptr()), front, static_cast<const int32_t *>(length.data_ptr()), (float)scale, scratch, (size_t)ws.numel(),
                       own, to, stream);
    }));
    check_waits(args[11], scratch, stream);
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// gemm_w4(A bf16 [R, K], codes uint8 [N, K / 2], scales bf16 [N, K / group], out or None, workspace or None)
PyObject *gemm_w4(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 5);
    const at::Tensor &a = dims(typed(args[0], "A", at::kBFloat16), "A", 2);
    const int64_t R = a.size(0), K = a.size(1);
    sized(a, "A", {R, K});
    const at::Tensor &codes = dims(typed(args[1], "codes", at::kByte, &a), "codes", 2);
    const int64_t N = codes.size(0);
    sized(codes, "codes", {N, K / 2});
    const at::Tensor &scales = dims(typed(args[2], "scales", at::kBFloat16, &a), "scales", 2);
    const int64_t groups = scales.size(1);
    sized(scales, "scales", {N, groups});
    if (groups == 0 || K % groups) {
      PyErr_SetString(PyExc_ValueError, "scales: K is not a whole number of groups");
      throw Failed();
    }
    const int rows = count(R), k = count(K), cols = count(N), group = count(K / groups);
    const size_t need = gemm_w4_bytes_fn(rows, cols, k, group);
    if (need == 0) {
      PyErr_Format(error_class, "hsd_gemm_w4: unsupported shape R=%d N=%d K=%d, groups of %d", rows, cols, k, group);
      throw Failed();
    }
    const c10::cuda::CUDAGuard guard(a.device());
    at::Tensor out = args[3] == Py_None ? fresh({R, N}, at::kFloat) : sized(typed(args[3], "out", at::kFloat, &a), "out", {R, N});
    at::Tensor ws = args[4] == Py_None ? fresh({(int64_t)need}, at::kByte) : typed(args[4], "workspace", at::kByte, &a);
    if (!ws.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    void *pa = a.data_ptr(), *pc = codes.data_ptr(), *ps = scales.data_ptr(), *scratch = ws.data_ptr(), *stream = current_stream();
    float *to = static_cast<float *>(out.data_ptr());
    check(released([&] { return gemm_w4_fn(pa, rows, k, pc, ps, cols, group, to, scratch, (size_t)ws.numel(), stream); }));
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// quantize_rows(x [rows, K])
PyObject *quantize_rows(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 1);
    const at::Tensor &x = dims(tensor(args[0]), "x", 2);
    const at::ScalarType source = cache_type(x, "x");
    typed(args[0], "x", source);
    if (x.size(1) > 1 && x.stride(1) != 1) refuse("x: the values of a row have to be contiguous");
    const int rows = count(x.size(0)), k = count(x.size(1));
    const long long stride = rows > 1 ? x.stride(0) : k;
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor codes = fresh({rows, k}, at::kChar), scales = fresh({rows}, at::kFloat);
    void *from = x.data_ptr(), *to = codes.data_ptr(), *stream = current_stream();
    float *scale = static_cast<float *>(scales.data_ptr());
    check(released([&] { return quantize_fn(from, source == at::kFloat ? HSD_F32 : HSD_BF16, rows, k, stride, to, scale, stream); }));
    PyObject *first = THPVariable_Wrap(std::move(codes)), *second = THPVariable_Wrap(std::move(scales)), *both = nullptr;
    if (first && second) both = PyTuple_Pack(2, first, second);
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// gemm_w8(A [R, K], codes int8 [N, K], scales fp32 [N], out dtype, a_scales fp32 [R] or None, out or None, workspace or None, check)
PyObject *gemm_w8(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 8);
    const at::Tensor &a = dims(tensor(args[0]), "A", 2);
    const bool coded = a.scalar_type() == at::kChar;
    const at::ScalarType source = coded ? at::kChar : cache_type(a, "A");
    typed(args[0], "A", source);
    const int64_t R = a.size(0), K = a.size(1);
    sized(a, "A", {R, K});
    const at::Tensor &codes = dims(typed(args[1], "codes", at::kChar, &a), "codes", 2);
    const int64_t N = codes.size(0);
    sized(codes, "codes", {N, K});
    const at::Tensor &scales = sized(typed(args[2], "scales", at::kFloat, &a), "scales", {N});
    if (!THPDtype_Check(args[3])) {
      PyErr_SetString(PyExc_TypeError, "out_dtype: expected a torch.dtype");
      throw Failed();
    }
    const at::ScalarType to_type = reinterpret_cast<THPDtype *>(args[3])->scalar_type;
    if (to_type != at::kFloat && to_type != at::kBFloat16) refuse("out_dtype: expected float32 or bfloat16");
    if (coded != (args[4] != Py_None)) refuse("a_scales go with an A of int8, and with no other");
    const float *row_scales = coded ? static_cast<const float *>(sized(typed(args[4], "a_scales", at::kFloat, &a), "a_scales", {R}).data_ptr()) : nullptr;
    const int rows = count(R), k = count(K), cols = count(N), dtype = coded ? HSD_I8 : source == at::kFloat ? HSD_F32 : HSD_BF16;
    const size_t need = gemm_w8_bytes_fn(dtype, rows, cols, k);
    if (need == 0) {
      PyErr_Format(error_class, "hsd_gemm_w8: unsupported shape R=%d N=%d K=%d", rows, cols, k);
      throw Failed();
    }
    const c10::cuda::CUDAGuard guard(a.device());
    at::Tensor out = args[5] == Py_None ? fresh({R, N}, to_type) : sized(typed(args[5], "out", to_type, &a), "out", {R, N});
    at::Tensor ws = args[6] == Py_None ? fresh({(int64_t)need}, at::kByte) : typed(args[6], "workspace", at::kByte, &a);
    if (!ws.is_contiguous()) refuse("expected a contiguous CUDA tensor");
    void *pa = a.data_ptr(), *pc = codes.data_ptr(), *to = out.data_ptr(), *scratch = ws.data_ptr(), *stream = current_stream();
    const float *col_scales = static_cast<const float *>(scales.data_ptr());
    check(released([&] {
      return gemm_w8_fn(pa, dtype, row_scales, rows, k, pc, col_scales, cols, to, to_type == at::kFloat ? HSD_F32 : HSD_BF16, scratch, (size_t)ws.numel(), stream);
    }));
    check_waits(args[7], scratch, stream);
    return THPVariable_Wrap(std::move(out));
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

// token_logprobs(logits [..., vocab], tokens int32 [...], top)
PyObject *token_logprobs(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    arguments(n, 3);
    const at::Tensor &logits = tensor(args[0]);
    if (logits.dim() < 1) {
      PyErr_SetString(PyExc_ValueError, "logits: expected a last dimension of tokens");
      throw Failed();
    }
    const int dtype = dtype_code(logits);
    void *from = device_data(logits);
    const at::IntArrayRef lead = logits.sizes().slice(0, logits.dim() - 1);
    const at::Tensor &tokens = sized(typed(args[1], "tokens", at::kInt, &logits), "tokens", lead);
    const int64_t top = PyLong_AsLongLong(args[2]);
    if (top == -1 && PyErr_Occurred()) throw Failed();
    if (top < 0) refuse("top: expected 0 or more");
    const int rows = count(tokens.numel()), vocab = count(logits.size(-1)), k = count(top);
    const c10::cuda::CUDAGuard guard(logits.device());
    std::vector<int64_t> more(lead.begin(), lead.end());
    more.push_back(top);
    at::Tensor out[5] = {fresh(lead, at::kFloat), fresh(lead, at::kFloat), fresh(lead, at::kInt), fresh(more, at::kInt), fresh(more, at::kFloat)};
    void *to[5], *stream = current_stream();
    for (int x = 0; x < 5; ++x) to[x] = out[x].data_ptr();
    check(released([&] {
      return logprobs_fn(from, dtype, rows, vocab, static_cast<const int32_t *>(tokens.data_ptr()), k, static_cast<float *>(to[0]), static_cast<float *>(to[1]),
                         static_cast<int32_t *>(to[2]), static_cast<int32_t *>(to[3]), static_cast<float *>(to[4]), stream);
    }));
    PyObject *all = PyTuple_New(5);
    if (!all) return nullptr;
    for (int x = 0; x < 5; ++x) {
      PyObject *o = THPVariable_Wrap(std::move(out[x]));
      if (!o) { Py_DECREF(all); return nullptr; }
      PyTuple_SET_ITEM(all, x, o);
    }
    return all;
  } catch (const Failed &) { return nullptr; }
  END_HANDLE_TH_ERRORS
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"init", FAST(init)}, {"draft_sample", FAST(draft_sample)}, {"verify_level", FAST(verify_level)},
                         {"gemm_bf16", FAST(gemm_bf16)}, {"kv_append", FAST(kv_append)}, {"kv_append_norm", FAST(kv_append_norm)}, {"quantize_rows", FAST(quantize_rows)}, {"gemm_w8", FAST(gemm_w8)}, {"prefix_attention", FAST(prefix_attention)},
                         {"paged_attention", FAST(paged_attention)},
                         {"gemm_w4", FAST(gemm_w4)}, {"token_logprobs", FAST(token_logprobs)}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls(void) { return PyModule_Create(&module); }
