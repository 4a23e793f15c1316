// The device-resident operators (include/horizonserve_device.h) on torch tensors: what device_ops.py calls.
//
// A captured loop pays for these checks once, a loop of single calls every time, and there they are most of a small operator's time: in Python they took
// 5 us of a call whose kernel takes 4.  So the checks, the description struct and the call are made here; device_ops.py keeps the signatures and
// turns a status into an exception.  Checks that fail raise ValueError.  No C++ exception leaves an entry point.
#include <Python.h>

#include <ATen/cuda/CUDAContextLight.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <limits>
#include <type_traits>

#include "../../include/horizonserve_device.h"

namespace {

struct Refused {};                                       // a Python exception is set
template <typename... A>
[[noreturn]] void refuse(const char* format, A... a) {
  PyErr_Format(PyExc_ValueError, format, a...);
  throw Refused{};
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse("%s: a tensor is wanted", what);
  return THPVariable_Unpack(o);
}
int device_of(const at::Tensor& t) { return t.is_cuda() ? int(t.get_device()) : -1; }
const char* name_of(at::ScalarType type) { return type == at::kInt ? "int32" : type == at::kFloat ? "fp32" : "uint8"; }

// Address of a contiguous tensor with n elements (any number if -1) on device d; NULL for None (the call refuses it where it is wanted).
template <typename T>
T* vec(PyObject* o, int64_t n, int d, const char* what) {
  constexpr at::ScalarType type = std::is_same<T, int32_t>::value ? at::kInt : at::kFloat;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || device_of(t) != d || !t.is_contiguous() || (n >= 0 && t.numel() != n)) {
    if (n < 0) refuse("%s: a contiguous %s tensor on device %d is wanted", what, name_of(type), d);
    refuse("%s: a contiguous %s tensor of %lld elements on device %d is wanted", what, name_of(type), static_cast<long long>(n), d);
  }
  return static_cast<T*>(t.data_ptr());
}
void* scratch(PyObject* o, int d) {
  const at::Tensor& t = tensor(o, "workspace");
  if (device_of(t) != d || !t.is_contiguous() || t.numel() * int64_t(t.element_size()) < int64_t(HS_DEVICE_WORKSPACE_BYTES))
    refuse("workspace: %u contiguous bytes on device %d are wanted", unsigned(HS_DEVICE_WORKSPACE_BYTES), d);
  return t.data_ptr();
}
int32_t int32(int64_t v, const char* what) {
  if (v < std::numeric_limits<int32_t>::min() || v > std::numeric_limits<int32_t>::max()) refuse("%s is out of range", what);
  return int32_t(v);
}
int32_t int32(PyObject* o, const char* what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return int32(int64_t(v), what);
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return v;
}
int type_of(const at::Tensor& t) {                       // HS_TYPE_*, or -1
  return t.scalar_type() == at::kFloat ? HS_TYPE_F32 : t.scalar_type() == at::kBFloat16 ? HS_TYPE_BF16 : t.scalar_type() == at::kHalf ? HS_TYPE_F16 : -1;
}

// [rows, heads, dim] with contiguous rows: its address, and the elements between rows.
void* rows(const at::Tensor& t, int64_t n, int64_t heads, int64_t dim, int d, const char* what, int64_t& stride) {
  if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != dim || device_of(t) != d || (t.stride(2) != 1 && dim != 1) ||
      (t.stride(1) != dim && heads != 1))
    refuse("%s: a [%lld, %lld, %lld] tensor with contiguous rows on device %d is wanted", what, static_cast<long long>(n), static_cast<long long>(heads),
           static_cast<long long>(dim), d);
  stride = n > 1 ? t.stride(0) : heads * dim;
  return t.data_ptr();
}
struct Pool {
  void* p;
  int device, type;
  int32_t layers, layer, pages, heads, dim;
};
Pool pool(PyObject* o, PyObject* layer) {
  const at::Tensor& t = tensor(o, "kv_pool");
  if (t.dim() != 6 || t.size(1) != 2 || t.size(4) != 16 || !t.is_contiguous()) refuse("kv_pool: a contiguous [layers, 2, pages, kv heads, 16, head_dim] tensor is wanted");
  Pool r;
  r.type = type_of(t);
  if (r.type != HS_TYPE_BF16 && r.type != HS_TYPE_F16) refuse("kv_pool: bf16 or fp16 is wanted");
  r.layer = int32(layer, "layer");
  if (r.layer < 0 || r.layer >= t.size(0)) refuse("layer is outside the pool");
  r.p = t.data_ptr();
  r.device = device_of(t);
  r.layers = int32(t.size(0), "layers");
  r.pages = int32(t.size(2), "pages");
  r.heads = int32(t.size(3), "kv heads");
  r.dim = int32(t.size(5), "head_dim");
  return r;
}
// The block tables of n requests, and the length of their rows.
int32_t* table_rows(PyObject* o, int64_t n, int d, int32_t& width) {
  const at::Tensor& t = tensor(o, "block_tables");
  if (t.dim() != 2 || t.size(0) != n) refuse("block_tables: one row per request is wanted");
  width = int32(t.size(1), "block_tables");
  return vec<int32_t>(o, -1, d, "block_tables");
}
float* rope_rows(PyObject* o, int d, int32_t& positions, int32_t& rotary_dim) {
  const at::Tensor& t = tensor(o, "table");
  if (t.dim() != 3 || t.size(2) != 2) refuse("table: [positions, pairs, 2] is wanted");
  positions = int32(t.size(0), "positions");
  rotary_dim = int32(2 * t.size(1), "rotary_dim");
  return vec<float>(o, -1, d, "table");
}

// The C entry points, as the library that the package has loaded gives them.
struct Entries {
  decltype(&hs_op_step_tables) step_tables;
  decltype(&hs_op_release_pages) release_pages;
  decltype(&hs_op_rope_table) rope_table;
  decltype(&hs_op_rope_cache) rope_cache;
  decltype(&hs_op_paged_attention) paged_attention;
  decltype(&hs_op_token_logprobs) token_logprobs;
} entries;

// One call on the current stream of device d, as the status.
template <typename A>
long call(hs_status_t (*fn)(const A*, int32_t, void*), const A& a, int d, PyObject* sm_budget) {
  if (d < 0) refuse("the operators work on CUDA tensors");
  if (!fn) refuse("the library is not bound");
  const int32_t budget = sm_budget == Py_None ? at::cuda::getDeviceProperties(c10::DeviceIndex(d))->multiProcessorCount : int32(sm_budget, "sm_budget");
  const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(d));
  void* stream = c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(d)).stream();
  PyThreadState* state = PyEval_SaveThread();
  const hs_status_t st = fn(&a, budget, stream);
  PyEval_RestoreThread(state);
  return long(st);
}

long step_tables(PyObject* const* o) {
  const at::Tensor& ctx = tensor(o[0], "ctx_len");
  const int d = device_of(ctx);
  const int64_t n = ctx.numel(), cap = tensor(o[7], "tok_seq").numel();
  hs_step_tables_t a{};
  a.n_seqs = int32(n, "requests");
  a.max_tokens = int32(cap, "tokens");
  a.ctx_len = vec<int32_t>(o[0], n, d, "ctx_len");
  a.q_len = vec<int32_t>(o[1], n, d, "q_len");
  a.free_list = vec<int32_t>(o[2], -1, d, "free_list");
  a.num_pages = int32(tensor(o[2], "free_list").numel(), "pages");
  a.free_count = vec<int32_t>(o[3], 1, d, "free_count");
  a.block_tables = table_rows(o[4], n, d, a.max_pages_per_seq);
  a.kv_len = vec<int32_t>(o[5], n, d, "kv_len");
  a.tok_begin = vec<int32_t>(o[6], n + 1, d, "tok_begin");
  a.tok_seq = vec<int32_t>(o[7], cap, d, "tok_seq");
  a.tok_pos = vec<int32_t>(o[8], cap, d, "tok_pos");
  a.tok_slot = vec<int32_t>(o[9], cap, d, "tok_slot");
  a.free_count_out = vec<int32_t>(o[10], 1, d, "free_count_out");
  a.workspace = scratch(o[11], d);
  a.status = vec<int32_t>(o[12], 1, d, "status");
  return call(entries.step_tables, a, d, o[13]);
}

long release_pages(PyObject* const* o) {
  const at::Tensor& ctx = tensor(o[1], "ctx_len");
  const int d = device_of(ctx);
  const int64_t n = ctx.numel();
  hs_release_pages_t a{};
  a.n_seqs = int32(n, "requests");
  a.done = vec<int32_t>(o[0], n, d, "done");
  a.ctx_len = vec<int32_t>(o[1], n, d, "ctx_len");
  a.block_tables = table_rows(o[2], n, d, a.max_pages_per_seq);
  a.free_list = vec<int32_t>(o[3], -1, d, "free_list");
  a.num_pages = int32(tensor(o[3], "free_list").numel(), "pages");
  a.free_count = vec<int32_t>(o[4], 1, d, "free_count");
  a.workspace = scratch(o[5], d);
  a.status = vec<int32_t>(o[6], 1, d, "status");
  return call(entries.release_pages, a, d, o[7]);
}

long rope_table(PyObject* const* o) {
  const int d = device_of(tensor(o[0], "table"));
  hs_rope_table_t a{};
  a.table = rope_rows(o[0], d, a.max_position, a.rotary_dim);
  a.base = number(o[1]);
  a.scaling = int32(o[2], "scaling");
  a.factor = number(o[3]);
  a.trained_positions = int32(o[4], "trained_positions");
  a.turns_slow = number(o[5]);
  a.turns_fast = number(o[6]);
  a.magnitude = number(o[7]);
  return call(entries.rope_table, a, d, o[8]);
}

long rope_cache(PyObject* const* o) {
  const Pool kv = pool(o[7], o[8]);
  const at::Tensor &q = tensor(o[0], "q"), &k = tensor(o[1], "k"), &v = tensor(o[2], "v"), &q_out = tensor(o[6], "q_out");
  const int d = kv.device, src = type_of(q);
  if (src < 0 || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) refuse("q, k, v: one of fp32, bf16, fp16 is wanted");
  if (type_of(q_out) != kv.type) refuse("q_out: the pool's type is wanted");
  if (q.dim() != 3) refuse("q: [tokens, heads, head_dim] is wanted");
  const int64_t n = q.size(0), hq = q.size(1);
  hs_rope_cache_t a{};
  a.n_tokens = int32(n, "tokens");
  a.n_q_heads = int32(hq, "query heads");
  a.n_kv_heads = kv.heads;
  a.head_dim = kv.dim;
  a.src_type = src;
  a.cache_type = kv.type;
  a.q = rows(q, n, hq, kv.dim, d, "q", a.q_stride);
  a.k = rows(k, n, kv.heads, kv.dim, d, "k", a.k_stride);
  a.v = rows(v, n, kv.heads, kv.dim, d, "v", a.v_stride);
  a.q_out = rows(q_out, n, hq, kv.dim, d, "q_out", a.q_out_stride);
  a.tok_pos = vec<int32_t>(o[3], n, d, "tok_pos");
  a.tok_slot = vec<int32_t>(o[4], n, d, "tok_slot");
  a.table = rope_rows(o[5], d, a.max_position, a.rotary_dim);
  a.n_layers = kv.layers;
  a.layer = kv.layer;
  a.num_pages = kv.pages;
  a.kv_pool = kv.p;
  a.status = vec<int32_t>(o[9], 1, d, "status");
  a.interleaved = PyObject_IsTrue(o[10]);
  if (a.interleaved < 0) throw Refused{};
  return call(entries.rope_cache, a, d, o[11]);
}

long paged_attention(PyObject* const* o) {
  const Pool kv = pool(o[1], o[2]);
  const at::Tensor &q = tensor(o[0], "q"), &out = tensor(o[5], "o");
  const int d = kv.device;
  if (type_of(q) != kv.type || type_of(out) != kv.type) refuse("q, o: the pool's type is wanted");
  if (q.dim() != 3) refuse("q: [tokens, heads, head_dim] is wanted");
  const int64_t t = q.size(0), hq = q.size(1), n = tensor(o[4], "kv_len").numel();
  hs_paged_attention_t a{};
  a.n_seqs = int32(n, "requests");
  a.n_tokens = int32(t, "tokens");
  a.n_q_heads = int32(hq, "query heads");
  a.n_kv_heads = kv.heads;
  a.head_dim = kv.dim;
  a.type = kv.type;
  a.n_layers = kv.layers;
  a.layer = kv.layer;
  a.num_pages = kv.pages;
  a.q = rows(q, t, hq, kv.dim, d, "q", a.q_stride);
  a.kv_pool = kv.p;
  a.block_tables = table_rows(o[3], n, d, a.max_pages_per_seq);
  a.kv_len = vec<int32_t>(o[4], n, d, "kv_len");
  a.o = rows(out, t, hq, kv.dim, d, "o", a.o_stride);
  a.workspace = scratch(o[6], d);
  a.status = vec<int32_t>(o[7], 1, d, "status");
  a.lse = vec<float>(o[8], t * hq, d, "lse");
  a.tok_begin = vec<int32_t>(o[9], n + 1, d, "tok_begin");
  a.max_q_len = int32(o[10], "max_q_len");
  a.prefix_len = vec<int32_t>(o[11], n, d, "prefix_len");
  a.slopes = vec<float>(o[12], hq, d, "slopes");
  a.scale = o[13] == Py_None ? float(1.0 / std::sqrt(double(kv.dim))) : float(number(o[13]));
  a.cap = float(number(o[14]));
  a.window = int32(o[15], "window");
  return call(entries.paged_attention, a, d, o[16]);
}

long token_logprobs(PyObject* const* o) {
  const at::Tensor& x = tensor(o[0], "logits");
  const int d = device_of(x), type = type_of(x);
  if (type < 0 || x.dim() != 2 || (x.stride(1) != 1 && x.size(1) != 1)) refuse("logits: [rows, vocab] in fp32, bf16 or fp16 with contiguous rows is wanted");
  const int64_t n = x.size(0), v = x.size(1);
  hs_token_logprobs_t a{};
  a.n_rows = int32(n, "rows");
  a.vocab = int32(v, "vocab");
  a.type = type;
  a.logits = x.data_ptr();
  a.row_stride = n > 1 ? x.stride(0) : v;
  a.targets = vec<int32_t>(o[1], n, d, "targets");
  a.logprob = vec<float>(o[2], n, d, "logprob");
  a.workspace = scratch(o[3], d);
  a.status = vec<int32_t>(o[4], 1, d, "status");
  a.entropy = vec<float>(o[5], n, d, "entropy");
  a.rank = vec<int32_t>(o[6], n, d, "rank");
  if ((o[7] == Py_None) != (o[8] == Py_None)) refuse("top_ids and top_logprobs belong together");
  if (o[7] != Py_None) {
    const at::Tensor& ids = tensor(o[7], "top_ids");
    if (ids.dim() != 2 || ids.size(0) != n) refuse("top_ids and top_logprobs: [rows, alternatives] each are wanted");
    a.n_top = int32(ids.size(1), "alternatives");
    a.top_ids = vec<int32_t>(o[7], n * a.n_top, d, "top_ids");
    a.top_logprobs = vec<float>(o[8], n * a.n_top, d, "top_logprobs");
  }
  a.scale = float(number(o[9]));
  return call(entries.token_logprobs, a, d, o[10]);
}

// bind(addresses of the six C entry points in the order of Entries)
long bind(PyObject* const* o) {
  void* p[6];
  for (int i = 0; i < 6; ++i) {
    p[i] = PyLong_AsVoidPtr(o[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) refuse("an entry point is missing");
      throw Refused{};
    }
  }
  entries.step_tables = reinterpret_cast<decltype(entries.step_tables)>(p[0]);
  entries.release_pages = reinterpret_cast<decltype(entries.release_pages)>(p[1]);
  entries.rope_table = reinterpret_cast<decltype(entries.rope_table)>(p[2]);
  entries.rope_cache = reinterpret_cast<decltype(entries.rope_cache)>(p[3]);
  entries.paged_attention = reinterpret_cast<decltype(entries.paged_attention)>(p[4]);
  entries.token_logprobs = reinterpret_cast<decltype(entries.token_logprobs)>(p[5]);
  return 0;
}

template <long (*FN)(PyObject* const*), int ARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != ARGS) {
    PyErr_Format(PyExc_TypeError, "%d arguments are wanted", ARGS);
    return nullptr;
  }
  try {
    return PyLong_FromLong(FN(args));
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}
template <long (*FN)(PyObject* const*), int ARGS>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<FN, ARGS>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<bind, 6>("bind"),
                         method<step_tables, 14>("step_tables"),
                         method<release_pages, 8>("release_pages"),
                         method<rope_table, 9>("rope_table"),
                         method<rope_cache, 12>("rope_cache"),
                         method<paged_attention, 17>("paged_attention"),
                         method<token_logprobs, 11>("token_logprobs"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_device_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__device_binding() { return PyModule_Create(&module); }
