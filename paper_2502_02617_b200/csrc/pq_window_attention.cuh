// Attention of the last positions of every sequence over its paged 16-bit (or float32) window (included by pq_decode.cu).
//
// window_attention_kernel: a block of four warps takes up to kRows (query, head) rows of one kv head and a range of the
// window's tokens.  A warp reads a step of 8 or 16 tokens straight into registers, 16 bytes a lane, so that a row of keys
// lies in kLanes neighbouring lanes and the warp holds kGroups rows at a time; every group of lanes is a softmax stream of its
// own.  Scores: each lane multiplies its coordinates, and the sums of all (row, token) pairs are formed in one exchange that
// halves the values with every step (kVals values over kLanes lanes cost kVals - 1 shuffles, and each lane ends with one
// score).  The streams meet at the end: groups by shuffles, warps in shared memory, the blocks of a cluster in each other's
// shared memory, and the parts beyond a cluster in merge_attention_kernel.  Everything is float32 on the values as they are.
// bf16 rows of 64 and 128 are faster on tensor cores (pq_window_mma.cuh).  Bound by issue and the latency of its loads: float32
// windows of 32/8 heads of 128, 16 sequences of 2000 tokens 56 us (4.7 TB/s), one of 4000 18.8, six queries each on four of 2000 53.6 (93 in
// rows of four); in bf16, 64 sequences of up to 4096 tokens, it took 193 us against 111 there.
#pragma once

#include "pq_window_common.cuh"

namespace pq {

constexpr int kWinThreads = 128, kWinWarps = kWinThreads / 32, kWinMaxCluster = 8, kWinMaxParts = 16;

struct WindowArgs {
  int d, n_q_heads, n_kv_heads, n_q, io_dtype, out_dtype, row_blocks, n_parts;
  int n_splits;         // blocks that share a row block's tokens.  A row block's follow one another in the grid's first dimension, and so do the row
                        // blocks: the other dimensions end at 65535 (16384 positions of 64/8 heads are 65536 blocks of 16 rows)
  int early;            // the kernel ahead in the stream writes nothing that this one reads, and has every block say (launch_dependents)
                        // when all before it is done: wait for it at the end only, and use the SMs that it leaves idle
  int64_t n_rows;       // batch * n_q * n_q_heads: rows of q, out and of a part
  float scale;
  const void* q;
  const uint8_t* pool;
  const int32_t* lens;
  void* out;
  float* lse;           // optional
  float *part_out, *part_lse;   // n_parts > 1
  int32_t* status;
  Paging pg;
};

__device__ __forceinline__ float win_exp2(float x) { return exp2f(x); }
// exp2 of a difference of references: 0 from -inf on, 1 where nothing changes (also from -inf to -inf)
__device__ __forceinline__ float win_rescale(float from, float to) { return from == to ? 1.f : win_exp2(from - to); }

__device__ __forceinline__ float2 cluster_ld2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}

template <class T, int D, int kRows_>
struct WindowShape {
  static constexpr int kRows = kRows_;
  static constexpr int kC = 16 / sizeof(T);                // coordinates of a lane
  static constexpr int kLanes = D / kC;                    // lanes of a row
  static constexpr int kGroups = 32 / kLanes;              // rows of the warp at a time
  static constexpr int kTk = 16 / kGroups < 4 ? 16 / kGroups : 4;   // tokens of a group per step
  static constexpr int kStep = kTk * kGroups;              // tokens of a step: 4, 8 or 16, never across a page
  static constexpr int kVals = kRows * kTk;                // scores of a group per step
  static constexpr int kS = kVals > kLanes ? kVals / kLanes : 1;      // scores a lane ends with
  static constexpr int kDup = kVals < kLanes ? kLanes / kVals : 1;    // lanes with the same score
  static constexpr int kRl = kS > kTk ? kS / kTk : 1;                 // rows among a lane's scores
  static constexpr int kSr = kS / kRl;                                // scores of a row in a lane
  static constexpr int kRowLanes = kTk / kSr * kDup;                  // lanes with scores of the same row
  static_assert(kStep <= 16 && kLanes >= 2, "shape");
};

__device__ __forceinline__ uint4 win_load(const uint8_t* p, bool ok) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (ok) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// The 16 bytes of a lane as float32 pairs.
template <class T>
__device__ __forceinline__ void win_pairs(uint4 w, uint64_t* x) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f2_pack(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xFFFF0000u));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = f2_pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
  }
}

// The outputs o [stream][kRows][D] of a block's streams, relative to ml [stream][kRows] = (reference, denominator), merged into the
// first one's place.  True if there is a NaN among them; a barrier has passed at the end.
template <int D, int kThreads, int kStreams, int kRows>
__device__ __forceinline__ bool merge_streams(float* o, float2* ml, int n_rows) {
  bool nan = false;
  float2 merged = make_float2(-CUDART_INF_F, 0.f);   // of row tid
  const int tid = threadIdx.x;
  for (int i = tid; i < n_rows * D / 4; i += kThreads) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    float M = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < kStreams; ++w) M = fmaxf(M, ml[w * kRows + r].x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kStreams; ++w) {
      const float k = win_rescale(ml[w * kRows + r].x, M);
      const float4 v = *reinterpret_cast<const float4*>(o + (w * kRows + r) * D + c);
      acc = make_float4(fmaf(v.x, k, acc.x), fmaf(v.y, k, acc.y), fmaf(v.z, k, acc.z), fmaf(v.w, k, acc.w));
    }
    nan = nan || acc.x != acc.x || acc.y != acc.y || acc.z != acc.z || acc.w != acc.w;
    *reinterpret_cast<float4*>(o + r * D + c) = acc;
  }
  if (tid < n_rows) {
#pragma unroll
    for (int w = 0; w < kStreams; ++w) merged.x = fmaxf(merged.x, ml[w * kRows + tid].x);
#pragma unroll
    for (int w = 0; w < kStreams; ++w) merged.y = fmaf(ml[w * kRows + tid].y, win_rescale(ml[w * kRows + tid].x, merged.x), merged.y);
    nan = nan || merged.y != merged.y;
  }
  nan = __syncthreads_or(nan);
  if (tid < n_rows) ml[tid] = merged;
  __syncthreads();
  return nan;
}

// The last step of a block: the blocks of the cluster merge their outputs y [n_rows][D], relative to (reference, denominator) bl, and
// each block hands a share of them to store(row, first of four coordinates, the four, log-sum-exp).  Rows that have seen nothing, or
// only scores of -inf, are zeros and -inf.
template <int D, int kThreads, class Store>
__device__ __forceinline__ void cluster_merge(const float* y, const float2* bl, int n_rows, Store store) {
  uint32_t rank, n_blocks;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n_blocks));
  cluster_arrive();
  cluster_wait();
  const uint32_t y_at = (uint32_t)__cvta_generic_to_shared(y), bl_at = (uint32_t)__cvta_generic_to_shared(bl);
  for (int i = threadIdx.x + kThreads * rank; i < n_rows * D / 4; i += kThreads * n_blocks) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    float2 ml[kWinMaxCluster];
    float4 v[kWinMaxCluster];
#pragma unroll
    for (uint32_t k = 0; k < kWinMaxCluster; ++k) {   // all in flight at once
      ml[k] = make_float2(-CUDART_INF_F, 0.f);
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (k < n_blocks) {
        ml[k] = cluster_ld2(cluster_map(bl_at + r * 8, k));
        v[k] = cluster_ld4(cluster_map(y_at + (r * D + c) * 4, k));
      }
    }
    float M = -CUDART_INF_F, L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWinMaxCluster; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
    for (int k = 0; k < kWinMaxCluster; ++k) {   // block order: the result does not depend on who asks
      const float w = win_rescale(ml[k].x, M);
      L = fmaf(ml[k].y, w, L);
      acc = make_float4(fmaf(v[k].x, w, acc.x), fmaf(v[k].y, w, acc.y), fmaf(v[k].z, w, acc.z), fmaf(v[k].w, w, acc.w));
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    store(r, c, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv), L == 0.f ? -CUDART_INF_F : (M + log2f(L)) * 0.693147180559945309f);
  }
  cluster_arrive();   // nobody leaves while its shared memory may be read
  cluster_wait();
}
template <int D, class RowOf, class Seen>
__device__ __forceinline__ void window_finish(const WindowArgs& a, const float* y, const float2* bl, int n_rows, RowOf row_of, Seen seen) {
  uint32_t n_blocks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n_blocks));
  const int part = blockIdx.x % a.n_splits / n_blocks;
  cluster_merge<D, kWinThreads>(y, bl, n_rows, [&](int r, int c, const float4& acc, float lse) {
    const int64_t row = row_of(r), at = row * D + c;
    if (a.n_parts > 1) {
      *reinterpret_cast<float4*>(a.part_out + part * a.n_rows * D + at) = acc;
      if (c == 0) a.part_lse[part * a.n_rows + row] = lse;
    } else {
      if (a.out_dtype == PQ_DTYPE_BF16) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
        *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = acc;
      }
      if (c == 0 && a.lse != nullptr) a.lse[row] = lse;
    }
    if (c == 0 && a.lse == nullptr && part == 0 && seen(r) == 0) set_status(a.status, PQ_ERR_EMPTY);
  });
  if (a.early) asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void window_begin(const WindowArgs& a) {
  if (!a.early) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // behind the wait: see DecodeArgs::early
  }
}

// Sums of kN values over 2 kOff lanes: every exchange halves the values that a lane holds.
template <int kN, int kOff>
__device__ __forceinline__ void win_sum_lanes(float* s, int lane) {
  if constexpr (kOff > 0) {
    if constexpr (kN > 1) {
      const bool upper = (lane & kOff) != 0;
#pragma unroll
      for (int i = 0; i < kN / 2; ++i) {
        const float send = upper ? s[i] : s[i + kN / 2], keep = upper ? s[i + kN / 2] : s[i];
        s[i] = keep + __shfl_xor_sync(0xffffffffu, send, kOff);
      }
      win_sum_lanes<kN / 2, kOff / 2>(s, lane);
    } else {
      s[0] += __shfl_xor_sync(0xffffffffu, s[0], kOff);
      win_sum_lanes<1, kOff / 2>(s, lane);
    }
  }
}

template <class T, int D, int kRows>
__global__ void __launch_bounds__(kWinThreads) window_attention_kernel(const __grid_constant__ WindowArgs a) {
  using W = WindowShape<T, D, kRows>;
  constexpr int kC = W::kC, kP = kC / 2, kLanes = W::kLanes, kGroups = W::kGroups, kTk = W::kTk, kStep = W::kStep;
  constexpr int kVals = W::kVals, kS = W::kS, kRl = W::kRl, kSr = W::kSr;
  __shared__ __align__(16) float o_sm[kWinWarps][kRows][D];
  __shared__ __align__(16) float y_sm[kRows][D];            // the block's merged output, read by the cluster
  __shared__ float2 ml_sm[kWinWarps][kRows], bl_sm[kRows];  // (reference, denominator) of the warps and of the block
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, li = lane & (kLanes - 1), group = lane / kLanes;
  const int g = a.n_q_heads / a.n_kv_heads, hk = blockIdx.y, n_splits = a.n_splits, rb = blockIdx.x / n_splits, split = blockIdx.x % n_splits, b = blockIdx.z;
  const int r0 = rb * kRows, n_rows = min(kRows, a.n_q * g - r0);   // row r0 + r: query (r0 + r) / g, head hk * g + (r0 + r) % g
  window_begin(a);
  auto row_of = [&](int r) -> int64_t {   // of q, out and lse
    const int j = (r0 + r) / g;
    return ((int64_t)b * a.n_q + j) * a.n_q_heads + hk * g + (r0 + r - j * g);
  };
  const int len = min(max(__ldcg(a.lens + b), 0), a.pg.page_tokens * a.pg.pages_per_seq);
  auto seen = [&](int r) { return max(0, len - (a.n_q - 1 - (r0 + r) / g)); };
  const int most = seen(n_rows - 1), least = seen(0);
  // this block's range of the tokens: whole pieces of 16
  const int pieces = (most + 15) / 16;
  const int t_begin = (int)((int64_t)pieces * split / n_splits) * 16;
  const int t_end = min(most, (int)((int64_t)pieces * (split + 1) / n_splits) * 16);

  uint64_t q[kRows][kP], o[kRows][kP];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    float x[kC];
    const int64_t at = row_of(min(r, n_rows - 1)) * D + li * kC;
#pragma unroll
    for (int i = 0; i < kC; ++i) x[i] = tail_elem(a.q, a.io_dtype, at + i);
#pragma unroll
    for (int i = 0; i < kP; ++i) {
      q[r][i] = f2_pack(x[2 * i], x[2 * i + 1]);
      o[r][i] = 0ull;
    }
  }
  const float scale = a.scale * 1.4426950408889634f;   // scores in the log2 domain
  float m[kRl], l[kRl];
#pragma unroll
  for (int i = 0; i < kRl; ++i) {
    m[i] = -CUDART_INF_F;
    l[i] = 0.f;
  }
  const int j0 = li * kVals / kLanes;   // this lane's scores: j0 + s, row (j0 + s) / kTk, token (j0 + s) % kTk of the group

  // pages: a register of the warp holds the table's entries from `page0` on
  const int32_t* table = a.pg.table + (int64_t)b * a.pg.pages_per_seq;
  const int P = a.pg.page_tokens;
  const int64_t head_bytes = (int64_t)2 * P * D * sizeof(T), page_bytes = head_bytes * a.n_kv_heads;
  int t = t_begin + warp * kStep;   // the next step to request
  int page = t / P, slot = t - page * P, page0 = page;
  auto entries = [&](int first) {
    int e = 0;
    if ((int64_t)first * P + (int64_t)lane * P < t_end) e = __ldcg(table + first + lane);
    if ((unsigned)e >= (unsigned)a.pg.n_pages) {   // read page 0 instead: no address outside the pool is formed
      set_status(a.status, PQ_ERR_INVALID_ARG);
      e = 0;
    }
    return e;
  };
  int entry = entries(page0);
  auto step_at = [&]() -> const uint8_t* {   // where the keys of step t start for this lane
    if (page - page0 >= 32) entry = entries(page0 = page);
    const int64_t e = __shfl_sync(0xffffffffu, entry, page - page0);
    return a.pool + e * page_bytes + hk * head_bytes + (int64_t)(slot + group) * D * sizeof(T) + li * 16;
  };
  auto advance = [&]() {
    t += kWinWarps * kStep;
    slot += kWinWarps * kStep;
    while (slot >= P) {
      slot -= P;
      ++page;
    }
  };
  uint4 kbuf[kTk], vbuf[kTk];
  const int64_t v_off = (int64_t)P * D * sizeof(T);
  const uint8_t* src = nullptr;
  if (t < t_end) {
    src = step_at();
#pragma unroll
    for (int i = 0; i < kTk; ++i) kbuf[i] = win_load(src + i * kGroups * D * sizeof(T), t + i * kGroups + group < t_end);
#pragma unroll
    for (int i = 0; i < kTk; ++i) vbuf[i] = win_load(src + v_off + i * kGroups * D * sizeof(T), t + i * kGroups + group < t_end);
  }
  while (t < t_end) {
    const int t0 = t + group;   // token i of the group is t0 + i * kGroups
    const bool edge = t + kStep > least || t + kStep > t_end;   // some row does not see some token of the step
    float s[kVals];
#pragma unroll
    for (int i = 0; i < kTk; ++i) {
      uint64_t k[kP];
      win_pairs<T>(kbuf[i], k);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        uint64_t acc = f2_mul(q[r][0], k[0]);
#pragma unroll
        for (int c = 1; c < kP; ++c) acc = f2_fma(q[r][c], k[c], acc);
        float lo, hi;
        f2_unpack(acc, lo, hi);
        s[r * kTk + i] = lo + hi;
      }
    }
    advance();   // t is the step after this one
    if (t < t_end) {
      src = step_at();
#pragma unroll
      for (int i = 0; i < kTk; ++i) kbuf[i] = win_load(src + i * kGroups * D * sizeof(T), t + i * kGroups + group < t_end);
    }
    win_sum_lanes<kVals, kLanes / 2>(s, lane);   // of the lanes of a row
    float p[kS];
    bool grow = false;
#pragma unroll
    for (int i = 0; i < kS; ++i) {
      s[i] *= scale;
      if (edge) {
        const int tok = t0 + (j0 + i) % kTk * kGroups;
        if (tok >= t_end || tok >= seen(min((j0 + i) / kTk, n_rows - 1))) s[i] = -CUDART_INF_F;
      }
      grow = grow || s[i] > m[i / kSr] + 8.f || (m[i / kSr] == -CUDART_INF_F && s[i] > -CUDART_INF_F);
    }
    if (__any_sync(0xffffffffu, grow)) {   // the reference moves only when a score is well above it (p <= 2^8 otherwise)
      float corr[kRl];
#pragma unroll
      for (int i = 0; i < kRl; ++i) {
        float mx = m[i];
#pragma unroll
        for (int e = 0; e < kSr; ++e) mx = fmaxf(mx, s[i * kSr + e]);
#pragma unroll
        for (int off = 1; off < W::kRowLanes; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        corr[i] = win_rescale(m[i], mx);
        m[i] = mx;
        l[i] *= corr[i];
      }
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int j = r * kTk;
        const float c = __shfl_sync(0xffffffffu, corr[j / kSr % kRl], (lane & ~(kLanes - 1)) | (j * kLanes / kVals));
        const uint64_t c2 = f2_pack(c, c);
#pragma unroll
        for (int i = 0; i < kP; ++i) o[r][i] = f2_mul(o[r][i], c2);
      }
    }
#pragma unroll
    for (int i = 0; i < kS; ++i) {
      const float ref = m[i / kSr];
      p[i] = win_exp2(s[i] - (ref == -CUDART_INF_F ? 0.f : ref));   // nothing seen yet: every score is -inf
      l[i / kSr] += p[i];
    }
#pragma unroll
    for (int i = 0; i < kTk; ++i) {
      uint64_t v[kP];
      win_pairs<T>(vbuf[i], v);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int j = r * kTk + i;
        const float pr = __shfl_sync(0xffffffffu, p[j % kS], (lane & ~(kLanes - 1)) | (j * kLanes / kVals));
        // a value that the row does not see may be an infinity or a NaN
        if (edge && t0 + i * kGroups >= seen(min(r, n_rows - 1))) continue;
        const uint64_t p2 = f2_pack(pr, pr);
#pragma unroll
        for (int c = 0; c < kP; ++c) o[r][c] = f2_fma(p2, v[c], o[r][c]);
      }
    }
    if (t < t_end) {
#pragma unroll
      for (int i = 0; i < kTk; ++i) vbuf[i] = win_load(src + v_off + i * kGroups * D * sizeof(T), t + i * kGroups + group < t_end);
    }
  }

  // ---- the groups of the warp
#pragma unroll
  for (int i = 0; i < kRl; ++i) {
#pragma unroll
    for (int off = 1; off < W::kRowLanes; off <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
    l[i] *= 1.f / W::kDup;
    float mx = m[i];
#pragma unroll
    for (int off = kLanes; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    const float corr = win_rescale(m[i], mx);
    m[i] = mx;
    l[i] *= corr;
#pragma unroll
    for (int off = kLanes; off < 32; off <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
    if constexpr (kGroups > 1) {
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int j = r * kTk;
        if (j / kSr % kRl != i) continue;
        const float c = __shfl_sync(0xffffffffu, corr, (lane & ~(kLanes - 1)) | (j * kLanes / kVals));
        const uint64_t c2 = f2_pack(c, c);
#pragma unroll
        for (int k = 0; k < kP; ++k) o[r][k] = f2_mul(o[r][k], c2);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    float x[kC];
#pragma unroll
    for (int i = 0; i < kP; ++i) f2_unpack(o[r][i], x[2 * i], x[2 * i + 1]);
#pragma unroll
    for (int off = kLanes; off < 32; off <<= 1)
#pragma unroll
      for (int i = 0; i < kC; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], off);
    if (group == 0)
#pragma unroll
      for (int i = 0; i < kC; i += 4) *reinterpret_cast<float4*>(&o_sm[warp][r][li * kC + i]) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    const int j = r * kTk;
    if (group == 0 && li == j * kLanes / kVals) ml_sm[warp][r] = make_float2(m[j / kSr % kRl], l[j / kSr % kRl]);
  }
  __syncthreads();
  // ---- the warps of the block
  for (int i = tid; i < kRows * D / 4; i += kWinThreads) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    float M = -CUDART_INF_F, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWinWarps; ++w) M = fmaxf(M, ml_sm[w][r].x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWinWarps; ++w) {
      const float k = win_rescale(ml_sm[w][r].x, M);
      const float4 v = *reinterpret_cast<const float4*>(&o_sm[w][r][c]);
      L = fmaf(ml_sm[w][r].y, k, L);
      acc.x = fmaf(v.x, k, acc.x);
      acc.y = fmaf(v.y, k, acc.y);
      acc.z = fmaf(v.z, k, acc.z);
      acc.w = fmaf(v.w, k, acc.w);
    }
    *reinterpret_cast<float4*>(&y_sm[r][c]) = acc;
    if (c == 0) bl_sm[r] = make_float2(M, L);
  }
  window_finish<D>(a, &y_sm[0][0], bl_sm, n_rows, row_of, seen);
}

// How a window's tokens are cut among clusters of up to eight blocks, and parts beyond that.  An SM holds four blocks, and a block costs
// about 4 us beside its tiles of 16 tokens, of which each of its `streams` takes 0.9 us: one wave of blocks where that leaves a block two
// tiles at least, more where a block still has 16 tiles for every stream (uneven lengths then level out), and a merge kernel (2.5 us) only
// where a stream would have more than eight tiles.  us at 1, 2, 4, 8 splits, 32/8 heads: 16 sequences of 500 tokens 15.2, 13.7, 11.4, 16.8;
// of 2048 43, 35, 27, 31; 64 of 200 16, 21, 29, 50; 64 of 1024 to 4096 129, 119, 111, 121; one of 4096 66, 35, 20, 12.4 and in eight parts 11.1.
// Clusters of 3, 5, 6 and 7 where the wave stays a sixth below full: fuller ones no longer pack.  35 rows of eight sequences over 2048 tokens in
// clusters of 4 and 5 23.2, 20.8; 20 sequences of 600 in 2 and 3 16.5, 15.0; 12 of 2048 in 4, 5 and 6 23.2, 22.2, 29.1; 10 of 1000 in 4, 6 and 7 15.4, 14.3, 19.5.
struct WindowCut {
  int cluster, parts;
};
// `steps`: of a stream for a tile (float32 rows of 128 are read four tokens at a time, of 64 eight), each as long as a tile's otherwise.  Counted
// as tiles a float32 window of 4000 tokens stayed in one cluster: 43.6 us, 18.8 in parts.
static WindowCut cut_window(int64_t units, int max_len, int n_sm, int streams, int steps) {
  const int64_t tiles = ((int64_t)max_len + 15) / 16, one_wave = std::max<int64_t>(1, 4 * (int64_t)n_sm / units);
  const int64_t splits = std::min(std::max<int64_t>(1, tiles / 2), std::max(one_wave, tiles / (16 * streams)));
  WindowCut c = {1, 1};
  while (c.cluster < kWinMaxCluster && 2 * c.cluster <= splits) c.cluster *= 2;
  c.cluster = (int)std::max<int64_t>(c.cluster, std::min({splits, 10 * (int64_t)n_sm / (3 * units), (int64_t)kWinMaxCluster}));
  if (c.cluster == kWinMaxCluster)
    c.parts = (int)std::max<int64_t>(1, std::min({(tiles * steps + 64 * streams - 1) / (64 * streams), one_wave / kWinMaxCluster, (int64_t)kWinMaxParts}));
  return c;
}

static int32_t launch_window(void (*kernel)(WindowArgs), const WindowArgs& a, int batch, const WindowCut& cut, int smem, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.n_splits * a.row_blocks, a.n_kv_heads, batch);
  cfg.blockDim = dim3(kWinThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cut.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    cudaGetLastError();
    return PQ_ERR_CUDA;
  }
  return launch_status();
}
template <class T, int D>
static int32_t launch_window_rows(const WindowArgs& a, int rows, int batch, const WindowCut& cut, cudaStream_t stream) {
  return launch_window(rows == 1   ? window_attention_kernel<T, D, 1>
                       : rows == 2 ? window_attention_kernel<T, D, 2>
                       : rows == 4 ? window_attention_kernel<T, D, 4>
                                   : window_attention_kernel<T, D, 8>,
                       a, batch, cut, 0, stream);
}
}  // namespace pq
