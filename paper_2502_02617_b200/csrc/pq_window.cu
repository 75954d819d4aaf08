// The paged window of recent tokens: new rows on their way in, with the rotary position applied to queries and keys.  (The
// attention that reads it is pq_window_attention.cuh.)
#include <cmath>

#include "pq_common.cuh"
#include "pq_window_common.cuh"

namespace pq {

struct AppendArgs {
  int d, n_q_heads, n_kv_heads, batch, total_tokens, half, interleaved;   // half: pairs that are rotated
  int64_t q_token_stride, q_head_stride, kv_token_stride, kv_head_stride;
  const void *q, *k, *v;
  void *q_out, *pool;
  const double* frequencies;
  const int32_t *cu_seqlens, *offsets;
  int32_t *lens, *status;
  Paging pg;
};

// Where new row `token` goes: its sequence (batch: a row behind the last one), its place in the window, and the element of
// the pool where head 0's key starts (-1: not written).
struct AppendPlace {
  int seq, place;
  int64_t at;
};
__device__ __forceinline__ bool append_fits(const AppendArgs& a, int base, int count) {
  return base >= 0 && (int64_t)base + count <= (int64_t)a.pg.page_tokens * a.pg.pages_per_seq;
}
__device__ __forceinline__ int64_t append_target(const AppendArgs& a, int seq, int base, int count, int place) {
  if (!append_fits(a, base, count) || (unsigned)(place - base) >= (unsigned)count) {
    set_status(a.status, PQ_ERR_CAPACITY);
    return -1;
  }
  const int page = a.pg.table[(int64_t)seq * a.pg.pages_per_seq + place / a.pg.page_tokens];
  if ((unsigned)page >= (unsigned)a.pg.n_pages) {
    set_status(a.status, PQ_ERR_INVALID_ARG);
    return -1;
  }
  return window_row(a.pg, a.n_kv_heads, a.d, page, 0, 0, place % a.pg.page_tokens);
}
__device__ __forceinline__ AppendPlace append_place(const AppendArgs& a, int token) {
  AppendPlace p = {token, 0, -1};
  int first = token, count = 1;
  if (a.cu_seqlens != nullptr) {
    int lo = 0, hi = a.batch;   // the first sequence that ends behind the row
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.cu_seqlens[mid + 1] > token) hi = mid;
      else lo = mid + 1;
    }
    p.seq = lo;
    if (lo == a.batch) return p;
    first = a.cu_seqlens[lo];
    count = a.cu_seqlens[lo + 1] - first;
  }
  const int base = a.lens[p.seq];
  p.place = base + (token - first);
  p.at = append_target(a, p.seq, base, count, p.place);
  return p;
}
// Cosine and sine of position * frequency: a product of float64 loses nothing that matters at any position below 2^31, and
// what is left of a turn is small enough for float32.
__device__ __forceinline__ float2 rotary(int64_t position, double frequency) {
  double turns = (double)position * frequency * 0.15915494309189535;   // 1 / (2 pi)
  turns -= rint(turns);
  float2 cs;
  sincospif(2.f * (float)turns, &cs.y, &cs.x);
  return cs;
}

template <class T>
__device__ __forceinline__ float load_f32(const void* p, int64_t i) {
  return (float)reinterpret_cast<const T*>(p)[i];
}
template <class T>
__device__ __forceinline__ void store_f32(void* p, int64_t i, float v) {
  reinterpret_cast<T*>(p)[i] = (T)v;
}

// A thread takes a pair of elements of one head of one row, whatever the strides and alignments.
template <class T>
__global__ void __launch_bounds__(256) append_window_kernel(const __grid_constant__ AppendArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int pairs = a.d / 2, heads = a.n_q_heads + 2 * a.n_kv_heads;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / pairs;
  if (row >= (int64_t)a.total_tokens * heads) return;
  const int u = (int)(i % pairs), token = (int)(row / heads), head = (int)(row % heads);
  const AppendPlace p = append_place(a, token);
  if (p.seq >= a.batch) return;
  const bool is_q = head < a.n_q_heads, is_v = head >= a.n_q_heads + a.n_kv_heads;
  const int h = is_q ? head : is_v ? head - a.n_q_heads - a.n_kv_heads : head - a.n_q_heads;
  if (!is_q && p.at < 0) return;
  const void* src = is_q ? a.q : is_v ? a.v : a.k;
  const int64_t from = is_q ? token * a.q_token_stride + h * a.q_head_stride : token * a.kv_token_stride + h * a.kv_head_stride;
  void* dst = is_q ? a.q_out : a.pool;
  const int64_t to = is_q ? ((int64_t)token * a.n_q_heads + h) * a.d : p.at + (int64_t)(2 * h + (is_v ? 1 : 0)) * a.pg.page_tokens * a.d;
  const bool turn = !is_v && u < a.half;
  const int x = turn && !a.interleaved ? u : 2 * u, y = turn && !a.interleaved ? u + a.half : 2 * u + 1;   // copied pairs lie behind 2 * half
  const float vx = load_f32<T>(src, from + x), vy = load_f32<T>(src, from + y);
  if (turn) {
    const int64_t position = (int64_t)p.place + (a.offsets != nullptr ? a.offsets[p.seq] : 0);
    const float2 cs = rotary(position, a.frequencies[u]);
    store_f32<T>(dst, to + x, vx * cs.x - vy * cs.y);
    store_f32<T>(dst, to + y, vy * cs.x + vx * cs.y);
  } else {
    store_f32<T>(dst, to + x, vx);
    store_f32<T>(dst, to + y, vy);
  }
}

// The windows grow once their rows are in: a thread per sequence.
__global__ void __launch_bounds__(128) advance_windows_kernel(const __grid_constant__ AppendArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = blockIdx.x * 128 + threadIdx.x;
  if (b >= a.batch) return;
  const int base = a.lens[b], count = a.cu_seqlens != nullptr ? a.cu_seqlens[b + 1] - a.cu_seqlens[b] : 1;
  if (count <= 0 || !append_fits(a, base, count)) return;
  if (a.cu_seqlens != nullptr && a.cu_seqlens[b + 1] > a.total_tokens) {   // rows that do not exist
    set_status(a.status, PQ_ERR_INVALID_ARG);
    return;
  }
  for (int p = base / a.pg.page_tokens; p <= (base + count - 1) / a.pg.page_tokens; ++p)
    if ((unsigned)a.pg.table[(int64_t)b * a.pg.pages_per_seq + p] >= (unsigned)a.pg.n_pages) return;
  a.lens[b] = base + count;
}

static int32_t launch_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
  const int64_t work = (int64_t)a.total_tokens * (a.n_q_heads + 2 * a.n_kv_heads) * (a.d / 2);
  if (work > 0) {
    const dim3 grid((unsigned)((work + 255) / 256));
    const int32_t st = dtype == PQ_DTYPE_BF16 ? launch_dependent(append_window_kernel<__nv_bfloat16>, grid, 256, 0, stream, a)
                                              : launch_dependent(append_window_kernel<float>, grid, 256, 0, stream, a);
    if (st != PQ_OK) return st;
  }
  return launch_dependent(advance_windows_kernel, dim3((unsigned)((a.batch + 127) / 128)), 128, 0, stream, a);
}

}  // namespace pq

extern "C" {

int32_t pq_rotary_frequencies(int32_t rotary_dim, double theta, double* frequencies_host) {
  if (rotary_dim <= 0 || rotary_dim % 2 || !(theta > 0.0) || !std::isfinite(theta) || frequencies_host == nullptr) return PQ_ERR_INVALID_ARG;
  for (int i = 0; i < rotary_dim / 2; ++i) frequencies_host[i] = std::pow(theta, -2.0 * i / rotary_dim);
  return PQ_OK;
}

int64_t pq_window_bytes(int32_t head_dim, int32_t n_kv_heads, int32_t page_tokens, int32_t n_pages, int32_t dtype) {
  if (!pq::window_head_dim(head_dim) || (dtype != PQ_DTYPE_F32 && dtype != PQ_DTYPE_BF16)) return PQ_ERR_UNSUPPORTED;
  if (n_kv_heads <= 0 || page_tokens <= 0 || page_tokens % 16 || n_pages <= 0) return PQ_ERR_INVALID_ARG;
  const __int128 bytes = (__int128)n_pages * n_kv_heads * 2 * page_tokens * head_dim * (dtype == PQ_DTYPE_F32 ? 4 : 2);
  return bytes > ((__int128)1 << 62) ? (int64_t)PQ_ERR_UNSUPPORTED : (int64_t)bytes;
}

int32_t pq_append_window(int32_t head_dim, int32_t n_q_heads, int32_t n_kv_heads, const void* q_dev, const void* k_dev,
                         const void* v_dev, int32_t dtype, int64_t q_token_stride, int64_t q_head_stride,
                         int64_t kv_token_stride, int64_t kv_head_stride, const int32_t* cu_seqlens_dev, int32_t batch,
                         int32_t total_tokens, const double* frequencies_dev, int32_t rotary_dim, int32_t interleaved,
                         const int32_t* offsets_dev, void* q_out_dev, void* pool_dev, int32_t* window_lens_dev,
                         const pq_paging* paging, int32_t* status_dev, void* stream) {
  pq::NvtxRange nvtx_range("pq_append_window");
  if (!pq::window_head_dim(head_dim) || (dtype != PQ_DTYPE_F32 && dtype != PQ_DTYPE_BF16)) return PQ_ERR_UNSUPPORTED;
  if (!k_dev || !v_dev || !pool_dev || !window_lens_dev || !status_dev) return PQ_ERR_INVALID_ARG;
  if (batch <= 0 || total_tokens < 0 || n_kv_heads <= 0 || n_q_heads < 0) return PQ_ERR_INVALID_ARG;
  if ((q_dev != nullptr) != (n_q_heads > 0) || (q_out_dev != nullptr) != (n_q_heads > 0)) return PQ_ERR_INVALID_ARG;
  if (!cu_seqlens_dev && total_tokens != batch) return PQ_ERR_INVALID_ARG;
  if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 2 || (rotary_dim > 0) != (frequencies_dev != nullptr)) return PQ_ERR_INVALID_ARG;
  if (q_token_stride < 0 || q_head_stride < 0 || kv_token_stride < 0 || kv_head_stride < 0) return PQ_ERR_INVALID_ARG;
  pq::AppendArgs a;
  const int32_t st = pq::window_paging_from(paging, &a.pg);
  if (st != PQ_OK) return st;
  const int size = dtype == PQ_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)pool_dev & 15) || ((uintptr_t)frequencies_dev & 7) || (((uintptr_t)cu_seqlens_dev | (uintptr_t)offsets_dev | (uintptr_t)window_lens_dev | (uintptr_t)status_dev) & 3) ||
      (((uintptr_t)q_dev | (uintptr_t)k_dev | (uintptr_t)v_dev | (uintptr_t)q_out_dev) & (size - 1)))
    return PQ_ERR_ALIGNMENT;
  // a thread per pair of elements at most, in blocks of 256 whose number fits in 31 bits
  if ((__int128)total_tokens * ((int64_t)n_q_heads + 2 * (int64_t)n_kv_heads) * (head_dim / 2) >= (__int128)1 << 38) return PQ_ERR_UNSUPPORTED;
  a.d = head_dim; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.batch = batch; a.total_tokens = total_tokens;
  a.half = rotary_dim / 2; a.interleaved = interleaved != 0;
  a.q_token_stride = q_token_stride; a.q_head_stride = q_head_stride; a.kv_token_stride = kv_token_stride; a.kv_head_stride = kv_head_stride;
  a.q = q_dev; a.k = k_dev; a.v = v_dev; a.q_out = q_out_dev; a.pool = pool_dev; a.frequencies = frequencies_dev;
  a.cu_seqlens = cu_seqlens_dev; a.offsets = offsets_dev; a.lens = window_lens_dev; a.status = status_dev;
  return pq::launch_append(a, dtype, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
