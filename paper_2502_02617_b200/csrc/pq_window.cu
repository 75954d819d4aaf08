// The paged window of recent tokens: new rows on their way in, with the rotary position applied to queries and keys.  (The
// attention that reads it is pq_window_attention.cuh.)
#include <algorithm>
#include <climits>
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
  if (place < base || place - base >= count) {   // a row before the first sequence's, or ends that fall: no sequence's
    set_status(a.status, PQ_ERR_INVALID_ARG);
    return -1;
  }
  if (!append_fits(a, base, count)) {
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
// `seq`: a sequence at or before the row's.
__device__ __forceinline__ AppendPlace append_place(const AppendArgs& a, int token, int seq) {
  AppendPlace p = {seq, 0, -1};
  int first = token, count = 1;
  if (a.cu_seqlens != nullptr) {
    while (p.seq < a.batch && a.cu_seqlens[p.seq + 1] <= token) ++p.seq;   // the first sequence that ends behind the row
    if (p.seq >= a.batch) return p;
    first = a.cu_seqlens[p.seq];
    count = a.cu_seqlens[p.seq + 1] - first;
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

__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float2 bf16_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  const __nv_bfloat162 w = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&w);
}
// Elements e of x and of y are a pair, with the cosine and sine c[e] (bf16: c on 16 bytes).
template <class T>
__device__ __forceinline__ void turn_halves(uint4& x, uint4& y, const float2* c) {
  uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      const float2 p = bf16_pair(a[i]), q = bf16_pair(b[i]);
      const float4 k = *reinterpret_cast<const float4*>(c + 2 * i);
      a[i] = pair_bf16(p.x * k.x - q.x * k.y, p.y * k.z - q.y * k.w);
      b[i] = pair_bf16(q.x * k.x + p.x * k.y, q.y * k.z + p.y * k.w);
    } else {
      const float p = __uint_as_float(a[i]), q = __uint_as_float(b[i]);
      const float2 k = c[i];
      a[i] = __float_as_uint(p * k.x - q * k.y);
      b[i] = __float_as_uint(q * k.x + p * k.y);
    }
  }
  x = make_uint4(a[0], a[1], a[2], a[3]);
  y = make_uint4(b[0], b[1], b[2], b[3]);
}
// Neighbouring elements are a pair.
template <class T>
__device__ __forceinline__ uint4 turn_neighbours(const uint4& v, const float2* c) {
  uint32_t a[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = bf16_pair(a[i]), k = c[i];
      a[i] = pair_bf16(p.x * k.x - p.y * k.y, p.y * k.x + p.x * k.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float p = __uint_as_float(a[i]), q = __uint_as_float(a[i + 1]);
      const float2 k = c[i / 2];
      a[i] = __float_as_uint(p * k.x - q * k.y);
      a[i + 1] = __float_as_uint(q * k.x + p * k.y);
    }
  }
  return make_uint4(a[0], a[1], a[2], a[3]);
}

// The sequence that row `token` belongs to, or one before it.
__device__ __forceinline__ int sequence_of(const AppendArgs& a, int token) {
  if (a.cu_seqlens == nullptr) return token;
  int lo = 0, hi = a.batch;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.cu_seqlens[mid + 1] > token) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}
// A thread takes a pair of elements of one head of one row, whatever the strides and alignments.
template <class T>
__global__ void __launch_bounds__(256) append_window_kernel(const __grid_constant__ AppendArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int pairs = a.d / 2, heads = a.n_q_heads + 2 * a.n_kv_heads;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / pairs;
  if (row >= (int64_t)a.total_tokens * heads) return;
  const int u = (int)(i % pairs), token = (int)(row / heads), head = (int)(row % heads);
  const AppendPlace p = append_place(a, token, sequence_of(a, token));
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

// Whether a sequence's row pointers fall, or lie below row 0.  The look-ups above take them to rise: where they do not, the rows of a sequence by
// its own two ends are not the rows that were given to it, and a window that grew by them would hold rows nobody wrote.
__device__ __forceinline__ bool ends_fall(int first, int end) { return first < 0 || end < first; }
// A sequence's window grows by its rows, all of them or, where one of them has no place, none: its length after that, -1 where it stays.
// `first`, `end`: its row pointers (0 and 1 where every sequence has one row).
__device__ __forceinline__ int advanced_length(const AppendArgs& a, int b, int first, int end) {
  const int base = __ldcg(a.lens + b), count = end - first;
  if (count <= 0 || !append_fits(a, base, count)) return -1;
  if (a.cu_seqlens != nullptr && end > a.total_tokens) {   // rows that do not exist
    set_status(a.status, PQ_ERR_INVALID_ARG);
    return -1;
  }
  for (int p = base / a.pg.page_tokens; p <= (base + count - 1) / a.pg.page_tokens; ++p)
    if ((unsigned)__ldcg(a.pg.table + (int64_t)b * a.pg.pages_per_seq + p) >= (unsigned)a.pg.n_pages) return -1;
  return base + count;
}
// A thread per sequence, behind a kernel that has every block say (launch_dependents) when it has read the lengths: the windows
// grow while the rows are still on their way.  The wait at the end makes this kernel's end that of the rows' too.
__global__ void __launch_bounds__(128) advance_windows_kernel(const __grid_constant__ AppendArgs a) {
  const int b = blockIdx.x * 128 + threadIdx.x;
  int first = 0, end = 1, length = -1;
  bool falls = false;   // of any sequence: no window grows
  if (b < a.batch) {
    if (a.cu_seqlens != nullptr) {
      first = __ldcg(a.cu_seqlens + b);
      end = __ldcg(a.cu_seqlens + b + 1);
    }
    length = advanced_length(a, b, first, end);
    falls = ends_fall(first, end);
  }
  if (a.cu_seqlens != nullptr)
    for (int j = threadIdx.x; j < a.batch; j += 128)
      if (j != b) falls = falls || ends_fall(__ldcg(a.cu_seqlens + j), __ldcg(a.cu_seqlens + j + 1));
  falls = __syncthreads_or(falls);
  if (length >= 0 && !falls) a.lens[b] = length;
  if (falls && threadIdx.x == 0) set_status(a.status, PQ_ERR_INVALID_ARG);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// The rows as 16-byte pieces, where they lie on 16 bytes and the rotated part of a head is a multiple of 32.  An item is two pieces of
// one head of one row: the two sides of kV rotated pairs, or copied elements.  A block takes kApItems items per thread of a few
// rows -- all loads go out before anything else --, looks up where its rows go, forms the cosines and sines of each row once for
// all heads, and stores.  Bound by HBM: 43456 rows of 32/8 heads of 128 in bf16 (1.07 GB in and out) 192 to 205 us, 5.2 to 5.6 TB/s; a thread per pair with
// its own cosine and sine took 1554.
constexpr int kApThreads = 256, kApItems = 3, kApTokens = 8, kApMaxHalf = 64;
template <class T>
__global__ void __launch_bounds__(kApThreads) append_window_pieces_kernel(const __grid_constant__ AppendArgs a, int tokens, int slices,
                                                                          bool alone) {
  constexpr int kV = 16 / sizeof(T);
  static_assert(kApMaxHalf * sizeof(float2) % 16 == 0, "turn_halves reads two pairs of a row at a time");
  __shared__ __align__(16) float2 cs[kApTokens][kApMaxHalf];
  __shared__ AppendPlace places[kApTokens];
  const int tid = threadIdx.x, token0 = blockIdx.x / slices * tokens, slice = blockIdx.x % slices;
  const int n_tokens = min(tokens, a.total_tokens - token0);
  const int per_head = a.d / (2 * kV), turns = a.half / kV, rest = (a.d - 2 * a.half) / 2;
  const int kv_items = a.n_kv_heads * per_head, q_items = a.n_q_heads * per_head, per_token = q_items + 2 * kv_items;
  const int first = slice * kApThreads * kApItems, n_items = min(n_tokens * per_token, first + kApThreads * kApItems);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  uint4 x[kApItems], y[kApItems];
  int token[kApItems], to[kApItems], gap[kApItems], turn[kApItems];   // to: element of the row's output (queries) or offset from AppendPlace::at
  bool is_q[kApItems];
#pragma unroll
  for (int k = 0; k < kApItems; ++k) {
    const int i = first + tid + k * kApThreads;
    token[k] = -1;
    if (i >= n_items) continue;
    const int t = i / per_token, r = i - t * per_token;
    is_q[k] = r < q_items;
    const bool is_v = r >= q_items + kv_items;
    const int rr = is_q[k] ? r : is_v ? r - q_items - kv_items : r - q_items, h = rr / per_head, u = rr - h * per_head;
    const bool rotated = !is_v && u < turns;
    const int u2 = is_v ? u : u - turns, behind = is_v ? 0 : 2 * a.half, half_rest = is_v ? a.d / 2 : rest;   // copied elements: two halves
    const int at = !rotated ? behind + u2 * kV : a.interleaved ? 2 * u * kV : u * kV;
    gap[k] = !rotated ? half_rest : a.interleaved ? kV : a.half;
    turn[k] = rotated ? u * kV : -1;
    token[k] = t;
    const T* src = reinterpret_cast<const T*>(is_q[k] ? a.q : is_v ? a.v : a.k) +
                   (is_q[k] ? (token0 + t) * a.q_token_stride + h * a.q_head_stride : (token0 + t) * a.kv_token_stride + h * a.kv_head_stride) + at;
    to[k] = is_q[k] ? h * a.d + at : (2 * h + (is_v ? 1 : 0)) * a.pg.page_tokens * a.d + at;
    x[k] = ld_once(src);
    y[k] = ld_once(src + gap[k]);
  }
  bool falls = false;
  if (a.cu_seqlens != nullptr) {   // the sequence of the block's first row: as many as end at it or before
    int seq = 0;
    for (int j = 0; j < a.batch; j += kApThreads) {
      const bool is = j + tid < a.batch;
      const int first = is ? a.cu_seqlens[j + tid] : 0, end = is ? a.cu_seqlens[j + tid + 1] : INT_MAX;
      falls = falls || ends_fall(first, end);
      seq += __syncthreads_count(end <= token0);
    }
    if (tid < n_tokens) places[tid] = append_place(a, token0 + tid, seq);
  } else if (tid < n_tokens) {
    places[tid] = append_place(a, token0 + tid, token0 + tid);
  }
  falls = __syncthreads_or(falls);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // this block has read the lengths
  if (alone) {   // nobody else reads them
    if (a.cu_seqlens == nullptr) {
      if (tid < n_tokens) {
        const int length = advanced_length(a, token0 + tid, 0, 1);
        if (length >= 0) a.lens[token0 + tid] = length;
      }
    } else if (falls) {
      if (tid == 0) set_status(a.status, PQ_ERR_INVALID_ARG);
    } else {
      for (int b = tid; b < a.batch; b += kApThreads) {
        const int length = advanced_length(a, b, __ldcg(a.cu_seqlens + b), __ldcg(a.cu_seqlens + b + 1));
        if (length >= 0) a.lens[b] = length;
      }
    }
  }
  for (int i = tid; i < n_tokens * a.half; i += kApThreads) {
    const int t = i / a.half, u = i - t * a.half;
    const AppendPlace p = places[t];
    if (p.seq < a.batch) cs[t][u] = rotary((int64_t)p.place + (a.offsets != nullptr ? a.offsets[p.seq] : 0), a.frequencies[u]);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kApItems; ++k) {
    if (token[k] < 0) continue;
    const AppendPlace p = places[token[k]];
    if (p.seq >= a.batch || (!is_q[k] && p.at < 0)) continue;
    if (turn[k] >= 0) {
      const float2* c = &cs[token[k]][turn[k]];
      if (a.interleaved) {
        x[k] = turn_neighbours<T>(x[k], c);
        y[k] = turn_neighbours<T>(y[k], c + kV / 2);
      } else {
        turn_halves<T>(x[k], y[k], c);
      }
    }
    T* dst = is_q[k] ? reinterpret_cast<T*>(a.q_out) + (int64_t)(token0 + token[k]) * a.n_q_heads * a.d + to[k]
                     : reinterpret_cast<T*>(a.pool) + p.at + to[k];
    *reinterpret_cast<uint4*>(dst) = x[k];
    *reinterpret_cast<uint4*>(dst + gap[k]) = y[k];
  }
}

template <class T>
static int32_t launch_append_as(const AppendArgs& a, cudaStream_t stream) {
  constexpr int kV = 16 / sizeof(T);
  const int heads = a.n_q_heads + 2 * a.n_kv_heads;
  bool advanced = false;
  auto on16 = [](const void* p, int64_t s0, int64_t s1) { return ((uintptr_t)p & 15) == 0 && s0 * (int64_t)sizeof(T) % 16 == 0 && s1 * (int64_t)sizeof(T) % 16 == 0; };
  const bool pieces = a.half % kV == 0 && (int64_t)2 * a.n_kv_heads * a.pg.page_tokens * a.d < (1ll << 31) && on16(a.k, a.kv_token_stride, a.kv_head_stride) && on16(a.v, 0, 0) &&
                      on16(a.q, a.q_token_stride, a.q_head_stride) && on16(a.q_out, 0, 0);
  if (a.total_tokens > 0 && pieces) {
    const int64_t per_token = (int64_t)heads * a.d / (2 * kV), most = kApThreads * kApItems;
    const int slices = (int)((per_token + most - 1) / most);
    const int tokens = (int)(slices > 1 ? 1 : std::min<int64_t>(kApTokens, most / per_token));
    const dim3 grid((unsigned)(((int64_t)a.total_tokens + tokens - 1) / tokens * slices));
    // every row's length is read by one block only, and either no other block's rows belong to the same sequence or there is no other
    const bool alone = slices == 1 && (a.cu_seqlens == nullptr || grid.x == 1);
    const int32_t st = launch_dependent(append_window_pieces_kernel<T>, grid, kApThreads, 0, stream, a, tokens, slices, alone);
    if (st != PQ_OK) return st;
    advanced = alone;
  } else if (a.total_tokens > 0) {
    const int64_t work = (int64_t)a.total_tokens * heads * (a.d / 2);
    const int32_t st = launch_dependent(append_window_kernel<T>, dim3((unsigned)((work + 255) / 256)), 256, 0, stream, a);
    if (st != PQ_OK) return st;
  } else {
    return PQ_OK;
  }
  return advanced ? PQ_OK : launch_dependent(advance_windows_kernel, dim3((unsigned)((a.batch + 127) / 128)), 128, 0, stream, a);
}

static int32_t launch_append(const AppendArgs& a, int dtype, cudaStream_t stream) {
  return dtype == PQ_DTYPE_BF16 ? launch_append_as<__nv_bfloat16>(a, stream) : launch_append_as<float>(a, stream);
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
  if (!pool_dev || !window_lens_dev || !status_dev || (total_tokens != 0 && (!k_dev || !v_dev))) return PQ_ERR_INVALID_ARG;
  if (batch <= 0 || total_tokens < 0 || n_kv_heads <= 0 || n_q_heads < 0) return PQ_ERR_INVALID_ARG;
  if (total_tokens > 0 && ((q_dev != nullptr) != (n_q_heads > 0) || (q_out_dev != nullptr) != (n_q_heads > 0))) return PQ_ERR_INVALID_ARG;
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
