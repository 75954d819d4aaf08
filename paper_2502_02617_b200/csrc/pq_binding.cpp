// The calls of a serving loop (encode, append, the attention calls) from Python tensors to the C ABI without ctypes: one
// vectorcall per entry point that checks shapes and dtypes, reads the data pointers and the current stream, and calls the
// library.  A ctypes call with seventeen arguments, its pointer conversions and the stream lookup cost 8 to 10 us, more
// than the kernels of a short step; this path costs below 1 us.  Every function returns the library's status code.
//
// Arguments common to all: `stream` is None (PyTorch's current stream) or an object with a cuda_stream attribute,
// `paging` 0, the address of a struct pq_paging, or a tuple (page table tensor, tokens per page, pages of the pool).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/polarquant.h"

namespace {

struct PyError {};   // a Python exception has been set

[[noreturn]] void fail(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw PyError();
}
void check(bool ok, const char* text) {
  if (!ok) fail(PyExc_AssertionError, text);
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* tensor_or_none(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
template <class T = void>
T* ptr(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}
int32_t i32(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyError();
  if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, "value does not fit in 32 bits");
  return (int32_t)v;
}
float f32(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyError();
  return (float)v;
}
template <class T>
const T* address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw PyError();
  return static_cast<const T*>(p);
}
// The paging of a call, read before the interpreter lock is released.
class PagingArg {
 public:
  explicit PagingArg(PyObject* o) {
    if (o == Py_None) return;
    if (PyTuple_Check(o)) {
      check(PyTuple_GET_SIZE(o) == 3, "paging is (page table, tokens per page, pages)");
      const at::Tensor& table = tensor(PyTuple_GET_ITEM(o, 0));
      check(table.scalar_type() == at::kInt && table.is_contiguous() && table.dim() == 2, "the page table must be a contiguous int32 tensor [batch, pages]");
      paging_ = {ptr<int32_t>(table), i32(PyTuple_GET_ITEM(o, 1)), (int32_t)table.size(1), i32(PyTuple_GET_ITEM(o, 2))};
      paged_ = true;
    } else if (const auto* p = address<pq_paging>(o)) {
      paging_ = *p;
      paged_ = true;
    }
  }
  const pq_paging* get() const { return paged_ ? &paging_ : nullptr; }

 private:
  pq_paging paging_ = {};
  bool paged_ = false;
};
void* stream_of(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
  if (v == nullptr) throw PyError();
  void* p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (p == nullptr && PyErr_Occurred()) throw PyError();
  return p;
}
int32_t dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return PQ_DTYPE_F32;
  if (t.scalar_type() == at::kBFloat16) return PQ_DTYPE_BF16;
  fail(PyExc_TypeError, "unsupported dtype (float32 and bfloat16 are taken)");
}

// Calls the library without the interpreter lock, as ctypes does: a launch may block on a full queue, and the first call of a kernel loads
// it.  The arguments have been evaluated by then; the caller's frame holds the tensors.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <class... Params, class... Args>
int32_t call(int32_t (*fn)(Params...), Args... args) {
  const Unlocked unlocked;
  return fn(args...);
}

// Runs `body` with `n` arguments checked and every exception turned into a Python one.
template <class Body>
PyObject* entry(Py_ssize_t got, Py_ssize_t want, Body body) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return nullptr;
  }
  try {
    return PyLong_FromLong(body());
  } catch (const PyError&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

void check_rows(const at::Tensor& K, const at::Tensor& V) {   // packed rows [tokens, heads, d]
  check(K.dim() == 3 && V.sizes() == K.sizes() && V.scalar_type() == K.scalar_type() && K.stride(2) == 1 && V.strides() == K.strides(),
        "K and V must be [tokens, kv heads, head_dim] of one dtype with the same strides and contiguous vectors");
}
void check_query(const at::Tensor& q, const at::Tensor& out, int64_t dim) {
  check(q.dim() == dim && q.is_contiguous() && out.is_contiguous() && out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type(),
        "q and out must be contiguous tensors of one shape and dtype");
}

// encode(S, tables, K, V, cu_seqlens, cache, lens, capacity, status, paging, stream)
PyObject* encode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 11, [&]() -> int32_t {
    const at::Tensor &K = tensor(a[2]), &V = tensor(a[3]), &cu = tensor(a[4]);
    check_rows(K, V);
    const PagingArg paging(a[9]);
    const pq_paging* pg = paging.get();
    const int32_t d = (int32_t)K.size(2), h = (int32_t)K.size(1), total = (int32_t)K.size(0), batch = (int32_t)cu.numel() - 1;
    if (pg != nullptr)
      return call(pq_encode_kv_paged, d, h, ptr<float>(tensor(a[0])), ptr(tensor(a[1])), ptr(K), ptr(V), dtype_code(K), K.stride(0),
                                K.stride(1), ptr<int32_t>(cu), batch, total, ptr(tensor(a[5])), ptr<int32_t>(tensor(a[6])), pg,
                                ptr<int32_t>(tensor(a[8])), stream_of(a[10]));
    return call(pq_encode_kv, d, h, ptr<float>(tensor(a[0])), ptr(tensor(a[1])), ptr(K), ptr(V), dtype_code(K), K.stride(0), K.stride(1),
                        ptr<int32_t>(cu), batch, total, ptr(tensor(a[5])), ptr<int32_t>(tensor(a[6])), i32(a[7]),
                        ptr<int32_t>(tensor(a[8])), stream_of(a[10]));
  });
}

// append(S, tables, k_new, v_new, cache, lens, capacity, status, paging, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 10, [&]() -> int32_t {
    const at::Tensor &k = tensor(a[2]), &v = tensor(a[3]);
    check(k.dim() == 3 && k.is_contiguous() && v.is_contiguous() && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type(),
          "k_new and v_new must be contiguous [batch, kv heads, head_dim] of one dtype");
    const PagingArg paging(a[8]);
    const pq_paging* pg = paging.get();
    const int32_t d = (int32_t)k.size(2), h = (int32_t)k.size(1), batch = (int32_t)k.size(0);
    if (pg != nullptr)
      return call(pq_append_kv_paged, d, h, ptr<float>(tensor(a[0])), ptr(tensor(a[1])), ptr(k), ptr(v), dtype_code(k), batch,
                                ptr(tensor(a[4])), ptr<int32_t>(tensor(a[5])), pg, ptr<int32_t>(tensor(a[7])), stream_of(a[9]));
    return call(pq_append_kv, d, h, ptr<float>(tensor(a[0])), ptr(tensor(a[1])), ptr(k), ptr(v), dtype_code(k), batch, ptr(tensor(a[4])),
                        ptr<int32_t>(tensor(a[5])), i32(a[6]), ptr<int32_t>(tensor(a[7])), stream_of(a[9]));
  });
}

// attend(S, tables, q, cache, lens, n_kv_heads, capacity, max_len, scale, out, lse or None, workspace, status, paging, stream):
// q [batch, heads, d], or [batch, queries, heads, d] for the causal last positions of every sequence
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 15, [&]() -> int32_t {
    const at::Tensor &q = tensor(a[2]), &out = tensor(a[9]);
    const bool multi = q.dim() == 4;
    check_query(q, out, multi ? 4 : 3);
    const at::Tensor* lse = tensor_or_none(a[10]);
    const PagingArg paging(a[13]);
    const pq_paging* pg = paging.get();
    const int32_t d = (int32_t)q.size(-1), hq = (int32_t)q.size(-2), batch = (int32_t)q.size(0), hkv = i32(a[5]), cap = i32(a[6]),
                  most = i32(a[7]);
    const float scale = f32(a[8]);
    const float* S = ptr<float>(tensor(a[0]));
    const void *tables = ptr(tensor(a[1])), *cache = ptr(tensor(a[3]));
    const int32_t* lens = ptr<int32_t>(tensor(a[4]));
    void *ws = ptr(tensor(a[11])), *stream = stream_of(a[14]);
    int32_t* status = ptr<int32_t>(tensor(a[12]));
    if (lse != nullptr) {
      check(!multi && lse->scalar_type() == at::kFloat && lse->is_contiguous() && lse->dim() == 2 && lse->size(0) == batch && lse->size(1) == hq,
            "lse must be a contiguous float32 tensor [batch, query heads]");
      return call(pq_decode_attention_lse, d, hq, hkv, S, tables, ptr(q), dtype_code(q), cache, lens, batch, cap, pg, most, scale, ptr(out),
                                     ptr<float>(*lse), ws, status, stream);
    }
    if (multi) {
      const int32_t nq = (int32_t)q.size(1);
      if (pg != nullptr)
        return call(pq_multi_query_attention_paged, d, hq, hkv, S, tables, ptr(q), dtype_code(q), cache, lens, batch, nq, pg, most, scale,
                                              ptr(out), ws, status, stream);
      return call(pq_multi_query_attention, d, hq, hkv, S, tables, ptr(q), dtype_code(q), cache, lens, batch, nq, cap, most, scale, ptr(out),
                                      ws, status, stream);
    }
    if (pg != nullptr)
      return call(pq_decode_attention_paged, d, hq, hkv, S, tables, ptr(q), dtype_code(q), cache, lens, batch, pg, most, scale, ptr(out), ws,
                                       status, stream);
    return call(pq_decode_attention, d, hq, hkv, S, tables, ptr(q), dtype_code(q), cache, lens, batch, cap, most, scale, ptr(out), ws, status,
                               stream);
  });
}

// general_encode(cfg, S, boundaries, K, V, cu_seqlens, cache, lens, capacity, status, stream)
PyObject* general_encode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 11, [&]() -> int32_t {
    const at::Tensor &K = tensor(a[3]), &V = tensor(a[4]), &cu = tensor(a[5]);
    check_rows(K, V);
    const auto* cfg = address<pq_general_config>(a[0]);
    check(cfg != nullptr && K.size(2) == cfg->head_dim, "K and V must have the configuration's head_dim");
    return call(pq_general_encode_kv, cfg, (int32_t)K.size(1), ptr<float>(tensor(a[1])), ptr<double>(tensor(a[2])), ptr(K), ptr(V),
                                dtype_code(K), K.stride(0), K.stride(1), ptr<int32_t>(cu), (int32_t)cu.numel() - 1,
                                (int32_t)K.size(0), ptr(tensor(a[6])), ptr<int32_t>(tensor(a[7])), i32(a[8]),
                                ptr<int32_t>(tensor(a[9])), stream_of(a[10]));
  });
}

// general_attend(cfg, n_kv_heads, S, centroids, q, cache, lens, capacity, scale, out, status, stream)
PyObject* general_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 12, [&]() -> int32_t {
    const at::Tensor &q = tensor(a[4]), &out = tensor(a[9]);
    check(q.dim() == 3 && q.is_contiguous() && out.is_contiguous() && out.numel() >= q.numel() && out.scalar_type() == q.scalar_type(),
          "q must be [batch, heads, head_dim], out of its dtype with room for as many values, both contiguous");
    const auto* cfg = address<pq_general_config>(a[0]);
    check(cfg != nullptr && q.size(2) == cfg->head_dim, "q must have the configuration's head_dim");
    return call(pq_general_decode_attention, cfg, (int32_t)q.size(1), i32(a[1]), ptr<float>(tensor(a[2])), ptr<double>(tensor(a[3])), ptr(q),
                                       dtype_code(q), ptr(tensor(a[5])), ptr<int32_t>(tensor(a[6])), (int32_t)q.size(0), i32(a[7]),
                                       f32(a[8]), ptr(out), ptr<int32_t>(tensor(a[10])), stream_of(a[11]));
  });
}

// angle_histograms(S, K, V, hist, status, stream): hist int64 [levels, bins], counts are added
PyObject* angle_histograms(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> int32_t {
    const at::Tensor &K = tensor(a[1]), &V = tensor(a[2]), &hist = tensor(a[3]);
    check_rows(K, V);
    check(hist.scalar_type() == at::kLong && hist.is_contiguous() && hist.dim() == 2 && hist.size(0) == PQ_N_LEVELS,
          "hist must be a contiguous int64 tensor [levels, bins]");
    return call(pq_angle_histograms, (int32_t)K.size(2), (int32_t)K.size(1), ptr<float>(tensor(a[0])), ptr(K), ptr(V), dtype_code(K),
                               K.stride(0), K.stride(1), (int32_t)K.size(0), (int32_t)hist.size(1), ptr<uint64_t>(hist),
                               ptr<int32_t>(tensor(a[4])), stream_of(a[5]));
  });
}

// tail_attend(q, k_tail, v_tail, tail_lens, scale, out, lse or None, status, n_splits, stream)
PyObject* tail_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 10, [&]() -> int32_t {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &out = tensor(a[5]);
    const at::Tensor* lse = tensor_or_none(a[6]);
    const int32_t splits = i32(a[8]);
    check(q.dim() == 3 && q.is_contiguous() && out.is_contiguous() && out.scalar_type() == q.scalar_type(),
          "q and out must be contiguous tensors of one dtype");
    check(k.dim() == 4 && k.is_contiguous() && v.is_contiguous() && k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() &&
              k.size(0) == q.size(0) && k.size(3) == q.size(2),
          "the window must be contiguous [batch, tokens, kv heads, head_dim]");
    check(out.numel() == splits * q.numel() && (lse == nullptr || lse->numel() == splits * q.size(0) * q.size(1)),
          "out and lse must hold n_splits parts");
    return call(pq_tail_attention, (int32_t)q.size(2), (int32_t)q.size(1), (int32_t)k.size(2), ptr(q), dtype_code(q), ptr(k), ptr(v),
                             dtype_code(k), ptr<int32_t>(tensor(a[3])), (int32_t)q.size(0), (int32_t)k.size(1), splits, f32(a[4]),
                             ptr(out), lse == nullptr ? nullptr : ptr<float>(*lse), ptr<int32_t>(tensor(a[7])), stream_of(a[9]));
  });
}

// merge(parts_out, parts_lse, out, lse_out or None, status, stream)
PyObject* merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 6, [&]() -> int32_t {
    const at::Tensor &parts = tensor(a[0]), &lse = tensor(a[1]), &out = tensor(a[2]);
    const at::Tensor* lse_out = tensor_or_none(a[3]);
    check(parts.dim() == 4 && parts.is_contiguous() && lse.is_contiguous() && out.is_contiguous(), "contiguous tensors are taken");
    check(lse.scalar_type() == at::kFloat && lse.dim() == 3 && lse.sizes() == parts.sizes().slice(0, 3) &&
              out.sizes() == parts.sizes().slice(1, 3),
          "parts_out [parts, batch, heads, head_dim], parts_lse float32 [parts, batch, heads], out [batch, heads, head_dim]");
    return call(pq_merge_attention, (int32_t)parts.size(3), (int32_t)parts.size(2), (int32_t)parts.size(1), (int32_t)parts.size(0), ptr(parts),
                              dtype_code(parts), ptr<float>(lse), ptr(out), dtype_code(out),
                              lse_out == nullptr ? nullptr : ptr<float>(*lse_out), ptr<int32_t>(tensor(a[4])), stream_of(a[5]));
  });
}

// The device that all tensors of a call lie on.
c10::Device one_device(std::initializer_list<const at::Tensor*> tensors) {
  const at::Tensor* first = *tensors.begin();
  check(first->is_cuda(), "tensors on a CUDA device are taken");
  for (const at::Tensor* t : tensors) check(t == nullptr || t->device() == first->device(), "all tensors must be on one device");
  return first->device();
}
// Makes the tensors' device the current one for a call, whichever is current outside.
void* stream_on(const c10::Device& device, PyObject* o) {
  return o == Py_None ? c10::cuda::getCurrentCUDAStream(device.index()).stream() : stream_of(o);
}
const at::Tensor& int32s(PyObject* o, int64_t n, const char* text) {
  const at::Tensor& t = tensor(o);
  check(t.scalar_type() == at::kInt && t.is_contiguous() && t.numel() == n, text);
  return t;
}
// A pool of pages [page][kv head][K | V][token][head_dim] and the table behind `paging`.
struct PoolArg {
  const at::Tensor& pool;
  const PagingArg paging;
  PoolArg(PyObject* p, PyObject* pg, int64_t batch, int64_t d) : pool(tensor(p)), paging(pg) {
    check(PyTuple_Check(pg), "paging is (page table, tokens per page, pages)");
    const at::Tensor& table = tensor(PyTuple_GET_ITEM(pg, 0));
    check(pool.dim() == 5 && pool.is_contiguous() && pool.size(0) == paging.get()->n_pages && pool.size(2) == 2 &&
              pool.size(3) == paging.get()->page_tokens && pool.size(4) == d,
          "the pool must be a contiguous tensor [pages, kv heads, 2, tokens per page, head_dim]");
    check(table.size(0) == batch && table.device() == pool.device(), "the page table must name the pages of every sequence, on the pool's device");
  }
};

// append_window(q or None, k, v, cu_seqlens or None, frequencies or None, interleaved, offsets or None, q_out or None, pool, lens, status, paging,
//               stream)
PyObject* append_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 13, [&]() -> int32_t {
    const at::Tensor *q = tensor_or_none(a[0]), *freq = tensor_or_none(a[4]), *q_out = tensor_or_none(a[7]);
    const at::Tensor &k = tensor(a[1]), &v = tensor(a[2]), &lens = tensor(a[9]), &status = tensor(a[10]);
    check_rows(k, v);
    check(lens.scalar_type() == at::kInt && lens.is_contiguous() && lens.dim() == 1, "lens must be a contiguous int32 tensor [batch]");
    const int64_t batch = lens.size(0), total = k.size(0), d = k.size(2);
    const PoolArg pool(a[8], a[11], batch, d);
    check(pool.pool.scalar_type() == k.scalar_type() && pool.pool.size(1) == k.size(1), "k and v must have the pool's dtype and kv heads");
    check((q == nullptr) == (q_out == nullptr), "q and q_out go together");
    if (q != nullptr)
      check(q->dim() == 3 && q->size(0) == total && q->size(2) == d && q->stride(2) == 1 && q->scalar_type() == k.scalar_type() &&
                q_out->sizes() == q->sizes() && q_out->is_contiguous() && q_out->scalar_type() == q->scalar_type(),
            "q must be [tokens, heads, head_dim] with contiguous vectors, q_out contiguous, both of the rows' dtype");
    const at::Tensor* cu = a[3] == Py_None ? nullptr : &int32s(a[3], batch + 1, "cu_seqlens must be a contiguous int32 tensor [batch + 1]");
    const at::Tensor* offsets = a[6] == Py_None ? nullptr : &int32s(a[6], batch, "offsets must be a contiguous int32 tensor [batch]");
    check(freq == nullptr || (freq->scalar_type() == at::kDouble && freq->is_contiguous() && freq->dim() == 1), "frequencies must be a contiguous float64 tensor");
    check(status.scalar_type() == at::kInt && status.is_contiguous() && status.numel() >= PQ_STATUS_WORDS, "status must hold the status words");
    const c10::Device device = one_device({&k, &v, q, q_out, cu, offsets, freq, &lens, &status, &pool.pool});
    const c10::cuda::CUDAGuard guard(device);
    const int64_t rotary = freq == nullptr ? 0 : 2 * freq->size(0);
    check(rotary <= d && total <= INT32_MAX && batch <= INT32_MAX && k.size(1) <= INT32_MAX, "rotary dimensions within the head, sizes within 32 bits");
    const int interleaved = PyObject_IsTrue(a[5]);
    if (interleaved < 0) throw PyError();
    return call(pq_append_window, (int32_t)d, q == nullptr ? 0 : (int32_t)q->size(1), (int32_t)k.size(1), q == nullptr ? nullptr : ptr(*q), ptr(k), ptr(v),
                dtype_code(k), q == nullptr ? 0 : q->stride(0), q == nullptr ? 0 : q->stride(1), k.stride(0), k.stride(1),
                cu == nullptr ? nullptr : ptr<int32_t>(*cu), (int32_t)batch, (int32_t)total, rotary == 0 ? nullptr : ptr<double>(*freq), (int32_t)rotary,
                (int32_t)interleaved, offsets == nullptr ? nullptr : ptr<int32_t>(*offsets), q == nullptr ? nullptr : ptr(*q_out), ptr(pool.pool),
                ptr<int32_t>(lens), pool.paging.get(), ptr<int32_t>(status), stream_on(device, a[12]));
  });
}

// window_attend(q, pool, lens, max_len, scale, out, lse or None, workspace, status, paging, stream): q [batch, heads, d] or [batch, queries, heads, d]
PyObject* window_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 11, [&]() -> int32_t {
    const at::Tensor &q = tensor(a[0]), &out = tensor(a[5]), &ws = tensor(a[7]), &status = tensor(a[8]);
    const bool multi = q.dim() == 4;
    check_query(q, out, multi ? 4 : 3);
    const int64_t batch = q.size(0), n_q = multi ? q.size(1) : 1, hq = q.size(-2), d = q.size(-1);
    const PoolArg pool(a[1], a[9], batch, d);
    const at::Tensor& lens = int32s(a[2], batch, "lens must be a contiguous int32 tensor [batch]");
    const at::Tensor* lse = tensor_or_none(a[6]);
    check(lse == nullptr || (lse->scalar_type() == at::kFloat && lse->is_contiguous() && lse->sizes() == q.sizes().slice(0, q.dim() - 1)),
          "lse must be a contiguous float32 tensor of q's shape without the last dimension");
    check(status.scalar_type() == at::kInt && status.is_contiguous() && status.numel() >= PQ_STATUS_WORDS, "status must hold the status words");
    const int32_t most = i32(a[3]);
    check(batch <= INT32_MAX && n_q <= INT32_MAX && hq <= INT32_MAX, "sizes within 32 bits");
    const int64_t need = pq_window_workspace_bytes((int32_t)d, (int32_t)batch, (int32_t)n_q, (int32_t)hq, (int32_t)pool.pool.size(1), most);
    check(need < 0 || (ws.is_contiguous() && (int64_t)ws.nbytes() >= need), "the workspace is too small");   // below 0: the call itself says why
    const c10::Device device = one_device({&q, &out, lse, &ws, &status, &lens, &pool.pool});
    const c10::cuda::CUDAGuard guard(device);
    return call(pq_window_attention, (int32_t)d, (int32_t)hq, (int32_t)pool.pool.size(1), ptr(q), dtype_code(q), ptr(pool.pool), dtype_code(pool.pool),
                ptr<int32_t>(lens), (int32_t)batch, (int32_t)n_q, pool.paging.get(), most, f32(a[4]), ptr(out),
                lse == nullptr ? nullptr : ptr<float>(*lse), ptr(ws), ptr<int32_t>(status), stream_on(device, a[10]));
  });
}

// What prefix_attend and shared_attend have in common: (S, tables, q, cache, lens, seq, n_kv_heads, capacity, max_len, scale, out, workspace,
// status, paging, stream, ...); paging None (a contiguous cache of `capacity` tokens) or a tuple
struct PrefixArgs {
  const at::Tensor &S, &tables, &q, &cache, &lens, &out, &ws, &status;
  const PagingArg paging;
  int32_t seq, hkv, capacity, max_len;
  float scale;
  int32_t d, hq;
  explicit PrefixArgs(PyObject* const* a)
      : S(tensor(a[0])), tables(tensor(a[1])), q(tensor(a[2])), cache(tensor(a[3])), lens(tensor(a[4])), out(tensor(a[10])), ws(tensor(a[11])),
        status(tensor(a[12])), paging(a[13]), seq(i32(a[5])), hkv(i32(a[6])), capacity(i32(a[7])), max_len(i32(a[8])), scale(f32(a[9])) {
    check(q.dim() == 3 || q.dim() == 4, "q must be [batch, heads, head_dim] or [batch, queries, heads, head_dim]");
    check_query(q, out, q.dim());
    check(q.numel() <= INT32_MAX && q.numel() > 0, "queries within 31 bits of elements");
    d = (int32_t)q.size(-1);
    hq = (int32_t)q.size(-2);
    check(S.scalar_type() == at::kFloat && S.is_contiguous() && S.dim() == 2 && S.size(0) == d && S.size(1) == d, "S must be a float32 tensor [head_dim, head_dim]");
    check(lens.scalar_type() == at::kInt && lens.is_contiguous() && lens.dim() == 1, "lens must be a contiguous int32 tensor [batch]");
    check(ws.is_contiguous() && status.scalar_type() == at::kInt && status.is_contiguous() && status.numel() >= PQ_STATUS_WORDS, "workspace and status words");
    const pq_paging* pg = paging.get();
    const int64_t bytes = pg != nullptr ? pq_paged_cache_bytes(d, hkv, pg->page_tokens, pg->n_pages) : pq_cache_bytes(d, (int32_t)lens.size(0), hkv, capacity);
    check(bytes < 0 || (cache.is_contiguous() && (int64_t)cache.nbytes() >= bytes), "the cache is smaller than its sizes say");   // below 0: the call says why
    if (pg != nullptr) {
      check(PyTuple_Check(a[13]), "paging is (page table, tokens per page, pages)");
      const at::Tensor& table = tensor(PyTuple_GET_ITEM(a[13], 0));
      check(table.size(0) == lens.size(0) && table.device() == cache.device(), "the page table must have a row for every length, on the cache's device");
    }
  }
  int32_t queries() const { return (int32_t)(q.numel() / ((int64_t)d * hq)); }
};

// prefix_attend(..., lse or None): q of any number of queries, all of which see all tokens of sequence `seq` of the cache
PyObject* prefix_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 16, [&]() -> int32_t {
    const PrefixArgs p(a);
    const at::Tensor* lse = tensor_or_none(a[15]);
    check(lse == nullptr || (lse->scalar_type() == at::kFloat && lse->is_contiguous() && lse->sizes() == p.q.sizes().slice(0, p.q.dim() - 1)),
          "lse must be a contiguous float32 tensor of q's shape without the last dimension");
    const int64_t need = pq_prefix_workspace_bytes(p.d, p.queries(), p.hq, p.hkv, p.max_len);
    check(need < 0 || (int64_t)p.ws.nbytes() >= need, "the workspace is too small");   // below 0: the call itself says why
    const c10::Device device = one_device({&p.q, &p.S, &p.tables, &p.cache, &p.lens, &p.out, &p.ws, &p.status, lse});
    const c10::cuda::CUDAGuard guard(device);
    return call(pq_prefix_attention, p.d, p.hq, p.hkv, ptr<float>(p.S), ptr(p.tables), ptr(p.q), dtype_code(p.q), p.queries(), ptr(p.cache),
                ptr<int32_t>(p.lens), (int32_t)p.lens.size(0), p.seq, p.capacity, p.paging.get(), p.max_len, p.scale, ptr(p.out),
                lse == nullptr ? nullptr : ptr<float>(*lse), ptr(p.ws), ptr<int32_t>(p.status), stream_on(device, a[14]));
  });
}

// shared_attend(..., pool, window_lens, max_window, window_paging)
PyObject* shared_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return entry(n, 19, [&]() -> int32_t {
    const PrefixArgs p(a);
    const int32_t batch = (int32_t)p.q.size(0), n_q = p.q.dim() == 4 ? (int32_t)p.q.size(1) : 1, max_window = i32(a[17]);
    const PoolArg pool(a[15], a[18], batch, p.d);
    const at::Tensor& window_lens = int32s(a[16], batch, "the window's lens must be a contiguous int32 tensor [batch]");
    check(pool.pool.size(1) == p.hkv, "the window must have the cache's kv heads");
    const int64_t need = pq_shared_workspace_bytes(p.d, batch, n_q, p.hq, p.hkv, p.max_len, max_window);
    check(need < 0 || (int64_t)p.ws.nbytes() >= need, "the workspace is too small");
    const c10::Device device = one_device({&p.q, &p.S, &p.tables, &p.cache, &p.lens, &p.out, &p.ws, &p.status, &pool.pool, &window_lens});
    const c10::cuda::CUDAGuard guard(device);
    return call(pq_shared_attention, p.d, p.hq, p.hkv, ptr<float>(p.S), ptr(p.tables), ptr(p.q), dtype_code(p.q), batch, n_q, ptr(p.cache),
                ptr<int32_t>(p.lens), (int32_t)p.lens.size(0), p.seq, p.capacity, p.paging.get(), p.max_len, ptr(pool.pool), dtype_code(pool.pool),
                ptr<int32_t>(window_lens), pool.paging.get(), max_window, p.scale, ptr(p.out), ptr(p.ws), ptr<int32_t>(p.status),
                stream_on(device, a[14]));
  });
}

// current_stream(device index): the handle of PyTorch's current stream there
PyObject* current_stream(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    check(n == 1, "expected a device index");
    return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)i32(a[0])).stream());
  } catch (const PyError&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef kMethods[] = {
    {"current_stream", (PyCFunction)(void (*)(void))current_stream, METH_FASTCALL, nullptr},
    {"prefix_attend", (PyCFunction)(void (*)(void))prefix_attend, METH_FASTCALL, nullptr},
    {"shared_attend", (PyCFunction)(void (*)(void))shared_attend, METH_FASTCALL, nullptr},
    {"append_window", (PyCFunction)(void (*)(void))append_window, METH_FASTCALL, nullptr},
    {"window_attend", (PyCFunction)(void (*)(void))window_attend, METH_FASTCALL, nullptr},
    {"angle_histograms", (PyCFunction)(void (*)(void))angle_histograms, METH_FASTCALL, nullptr},
    {"tail_attend", (PyCFunction)(void (*)(void))tail_attend, METH_FASTCALL, nullptr},
    {"merge", (PyCFunction)(void (*)(void))merge, METH_FASTCALL, nullptr},
    {"encode", (PyCFunction)(void (*)(void))encode, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {"general_encode", (PyCFunction)(void (*)(void))general_encode, METH_FASTCALL, nullptr},
    {"general_attend", (PyCFunction)(void (*)(void))general_attend, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_pq_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pq_binding(void) { return PyModule_Create(&kModule); }
