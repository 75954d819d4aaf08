// Attention over the paged window on tensor cores: bf16 rows of 64 or 128 (included by pq_decode.cu).
//
// A block of four warps takes 16 kTiles (query, head) rows of a kv head and a range of the window's tokens.  kTiles (1 or 4) warps, each
// with 16 rows, share a stream of 16-token tiles; 4 / kTiles streams share the range.  A stream copies its tiles with 16-byte
// cp.async into a ring of its own, keys and values of a tile as one piece each, 16-byte chunk x of row t at x ^ (t & 7).
//   scores (rows x tokens) = Q (16 x D) K^T: bf16 queries as they are, float32 ones as three bf16 terms (24 bits)
//   output (rows x D) += P (16 x 16) V with the weights as two bf16 terms (their sum is off by 2^-17 at most)
// Products of bf16 are exact in float32 and summed there; scale and softmax are float32.
// A weight or term of 0 times an infinite value or key is a NaN that the row itself may not see: a block whose result holds a NaN
// is computed again, row by row, by window_again.
// Bound by HBM where there is enough of a window: 64 sequences of 1024 to 4096 tokens, 32/8 heads of 128, 713 MB in 111 us (6.4 TB/s); 16 of
// 2048 in 27 us.  Four blocks on an SM: with the query fragments in registers (166) and a ring of four pieces three fitted, and 64 sequences
// of 200 tokens took 22 us instead of 16.
#pragma once

namespace pq {

constexpr int kWmTile = 16, kWmRing = 3;
template <int D, int kQTerms, int kTiles>
struct WmShape {
  static constexpr int kStreams = kWinWarps / kTiles, kRows = 16 * kTiles;
  static constexpr int kPiece = kWmTile * D * 2, kRingBytes = kStreams * kWmRing * kPiece;
  static constexpr int kOut = kStreams * kRows * D * 4;        // the streams' outputs, where the ring was
  static constexpr int kMl = kRingBytes > kOut ? kRingBytes : kOut;   // (reference, denominator) [stream][row]
  static constexpr int kQ = kMl + kStreams * kRows * 8;        // queries: fragments [tile][term][k-step][lane]
  static constexpr int kBytes = kQ + kTiles * kQTerms * (D / 16) * 512;
};

// The rows of a block in float32, a warp at a time, whatever the values: y [rows][D] and ml as window_finish takes them.
template <int D>
__device__ __noinline__ void window_again(const WindowArgs& a, int b, int hk, int r0, int n_rows, int t_begin, int t_end, int len, float* y, float2* ml) {
  constexpr int kC = D / 32;
  const int lane = threadIdx.x & 31, g = a.n_q_heads / a.n_kv_heads, P = a.pg.page_tokens;
  for (int r = threadIdx.x >> 5; r < n_rows; r += kWinWarps) {
    const int j = (r0 + r) / g;
    const int64_t row = ((int64_t)b * a.n_q + j) * a.n_q_heads + hk * g + (r0 + r - j * g);
    const int end = min(t_end, len - (a.n_q - 1 - j));
    float q[kC], o[kC], m = -CUDART_INF_F, l = 0.f;
#pragma unroll
    for (int i = 0; i < kC; ++i) {
      q[i] = tail_elem(a.q, a.io_dtype, row * D + lane * kC + i);
      o[i] = 0.f;
    }
    for (int t = t_begin; t < end; ++t) {
      int page = a.pg.table[(int64_t)b * a.pg.pages_per_seq + t / P];
      if ((unsigned)page >= (unsigned)a.pg.n_pages) page = 0;
      const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(a.pool) + window_row(a.pg, a.n_kv_heads, D, page, hk, 0, t % P) + lane * kC;
      const __nv_bfloat16* v = k + (int64_t)P * D;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < kC; ++i) s = fmaf(q[i], __bfloat162float(k[i]), s);
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      s *= a.scale * 1.4426950408889634f;
      const float m_new = fmaxf(m, s), corr = win_rescale(m, m_new);
      m = m_new;
      const float p = win_exp2(s - (m == -CUDART_INF_F ? 0.f : m));
      l = l * corr + p;
#pragma unroll
      for (int i = 0; i < kC; ++i) o[i] = fmaf(p, __bfloat162float(v[i]), o[i] * corr);
    }
#pragma unroll
    for (int i = 0; i < kC; ++i) y[r * D + lane * kC + i] = o[i];
    if (lane == 0) ml[r] = make_float2(m, l);
  }
}

template <int D, int kQTerms, int kTiles>
__global__ void __launch_bounds__(kWinThreads, 4) window_mma_kernel(const __grid_constant__ WindowArgs a) {
  using W = WmShape<D, kQTerms, kTiles>;
  constexpr int kSteps = D / 16, kChunks = D / 8, kThreads = 32 * kTiles;   // threads of a stream
  extern __shared__ __align__(128) uint8_t wm_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, c4 = lane & 3;
  const int stream = warp / kTiles, tile = warp % kTiles, in_stream = tid % kThreads;
  const int g = a.n_q_heads / a.n_kv_heads, hk = blockIdx.y, n_splits = a.n_splits, rb = blockIdx.x / n_splits, split = blockIdx.x % n_splits, b = blockIdx.z;
  const int r0 = rb * W::kRows, n_rows = min(W::kRows, a.n_q * g - r0);   // row r0 + r: query (r0 + r) / g, head hk * g + (r0 + r) % g
  const uint32_t sm = (uint32_t)__cvta_generic_to_shared(wm_smem);
  window_begin(a);
  auto row_of = [&](int r) -> int64_t {   // of q, out and lse
    const int j = (r0 + r) / g;
    return ((int64_t)b * a.n_q + j) * a.n_q_heads + hk * g + (r0 + r - j * g);
  };
  const int P = a.pg.page_tokens;
  const int len = min(max(__ldcg(a.lens + b), 0), P * a.pg.pages_per_seq);
  auto seen = [&](int r) { return max(0, len - (a.n_q - 1 - (r0 + r) / g)); };
  const int most = seen(n_rows - 1), least = seen(0);
  const int pieces = (most + 15) / 16;
  const int t_begin = (int)((int64_t)pieces * split / n_splits) * 16;
  const int t_end = min(most, (int)((int64_t)pieces * (split + 1) / n_splits) * 16);
  const int n_tiles = (t_end - t_begin + kWmTile - 1) / kWmTile;
  const int mine = n_tiles > stream ? (n_tiles - stream + W::kStreams - 1) / W::kStreams : 0;   // tiles of this stream

  // ---- copies: piece 2k is the keys of the stream's tile k, 2k + 1 its values
  const uint32_t ring = sm + stream * (kWmRing * W::kPiece);
  const int32_t* table = a.pg.table + (int64_t)b * a.pg.pages_per_seq;
  int t_req = t_begin + stream * kWmTile, page = t_req / P, slot = t_req - page * P, page0 = page;
  auto entries = [&](int first) {   // a register of the warp holds the table's entries from `first` on
    int e = 0;
    if ((int64_t)first * P + (int64_t)lane * P < t_end) e = __ldcg(table + first + lane);
    if ((unsigned)e >= (unsigned)a.pg.n_pages) {   // read page 0 instead: no address outside the pool is formed
      set_status(a.status, PQ_ERR_INVALID_ARG);
      e = 0;
    }
    return e;
  };
  int entry = entries(page0);
  constexpr int kPass = kThreads / kChunks;   // rows of a pass of the stream's threads
  const int copy_row = in_stream / kChunks, copy_chunk = in_stream % kChunks;
  const uint8_t* src = nullptr;
  auto request = [&](int piece) {
    if (piece < 2 * mine) {
      if ((piece & 1) == 0) {
        if (page - page0 >= 32) entry = entries(page0 = page);
        const int64_t e = __shfl_sync(0xffffffffu, entry, page - page0);
        src = a.pool + ((e * a.n_kv_heads + hk) * 2 * P + slot + copy_row) * (D * 2) + copy_chunk * 16;
      }
      const uint8_t* from = src + (piece & 1) * (int64_t)P * (D * 2);
      const uint32_t dst = ring + (piece % kWmRing) * W::kPiece;
#pragma unroll
      for (int i = 0; i < kWmTile / kPass; ++i) {
        const int row = copy_row + i * kPass;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + row * (D * 2) + ((copy_chunk ^ (row & 7)) << 4)),
                     "l"(from + i * kPass * (D * 2)), "r"(t_req + row < t_end ? 16 : 0)
                     : "memory");
      }
      if (piece & 1) {
        t_req += W::kStreams * kWmTile;
        slot += W::kStreams * kWmTile;
        while (slot >= P) {
          slot -= P;
          ++page;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto sync_stream = [&]() {
    if constexpr (kTiles == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + stream), "n"(kThreads) : "memory");
  };
#pragma unroll
  for (int i = 0; i < kWmRing; ++i) request(i);

  // ---- queries: A operand of row g8 and g8 + 8 of the warp's tile (rows past the last repeat it)
  uint4* q_sm = reinterpret_cast<uint4*>(wm_smem + W::kQ) + tile * (kQTerms * kSteps * 32) + lane;
  {
    const int64_t row_lo = row_of(min(16 * tile + g8, n_rows - 1)) * D, row_hi = row_of(min(16 * tile + g8 + 8, n_rows - 1)) * D;
#pragma unroll
    for (int i = 0; i < kSteps / W::kStreams; ++i) {   // the streams share the work
      const int ks = stream + i * W::kStreams, k = 16 * ks + 2 * c4;
      if constexpr (kQTerms == 1) {
        const __nv_bfloat16* qp = reinterpret_cast<const __nv_bfloat16*>(a.q) + k;
        q_sm[ks * 32] = make_uint4(*reinterpret_cast<const uint32_t*>(qp + row_lo), *reinterpret_cast<const uint32_t*>(qp + row_hi),
                                   *reinterpret_cast<const uint32_t*>(qp + row_lo + 8), *reinterpret_cast<const uint32_t*>(qp + row_hi + 8));
      } else {
        const float* qp = reinterpret_cast<const float*>(a.q) + k;
        uint32_t w[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 v = *reinterpret_cast<const float2*>(qp + ((e & 1) ? row_hi : row_lo) + 8 * (e >> 1));
          bf16_terms(v.x, v.y, w[e]);
        }
#pragma unroll
        for (int term = 0; term < 3; ++term) q_sm[(term * kSteps + ks) * 32] = make_uint4(w[0][term], w[1][term], w[2][term], w[3][term]);
      }
    }
    __syncthreads();
  }

  const float scale = a.scale * 1.4426950408889634f;   // scores in the log2 domain
  float o[D / 8][4], m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};   // of rows g8 and g8 + 8; l: this lane's share
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  const int row_seen[2] = {seen(min(16 * tile + g8, n_rows - 1)), seen(min(16 * tile + g8 + 8, n_rows - 1))};
  const int k_row = (lane & 7) + ((lane >> 4) << 3), k_half = (lane >> 3) & 1;        // ldmatrix of keys: token, 8-coordinate half
  const int v_row = (lane & 7) + (((lane >> 3) & 1) << 3), v_half = lane >> 4;        // of values
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    const int t0 = t_begin + (stream + i * W::kStreams) * kWmTile;
    asm volatile("cp.async.wait_group %0;" ::"n"(kWmRing - 1) : "memory");
    sync_stream();
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};   // tokens t0 + 8 n + 2 c4, + 1 of rows g8 (0, 1) and g8 + 8 (2, 3)
    {
      const uint32_t at = ring + (2 * i % kWmRing) * W::kPiece + k_row * (D * 2);
#pragma unroll
      for (int ks = 0; ks < kSteps; ++ks) {
        uint32_t k4[4];
        ldmatrix_x4<false>(at + (((2 * ks + k_half) ^ (k_row & 7)) << 4), k4);
#pragma unroll
        for (int term = kQTerms - 1; term >= 0; --term) {   // small terms first
          const uint4 w = q_sm[(term * kSteps + ks) * 32];
          const uint32_t qa[4] = {w.x, w.y, w.z, w.w};
          mma_bf16_16816(s[0], qa, k4[0], k4[1]);
          mma_bf16_16816(s[1], qa, k4[2], k4[3]);
        }
      }
    }
    sync_stream();
    request(2 * i + kWmRing);   // takes the keys' place
    const bool edge = t0 + kWmTile > least || t0 + kWmTile > t_end;   // some row does not see some token of the tile
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[n][e] *= scale;
        if (edge) {
          const int t = t0 + 8 * n + 2 * c4 + (e & 1);
          if (t >= t_end || t >= row_seen[e >> 1]) s[n][e] = -CUDART_INF_F;
        }
      }
    float mx[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
    const bool grow = mx[0] > m[0] + 8.f || mx[1] > m[1] + 8.f || (m[0] == -CUDART_INF_F && mx[0] > m[0]) || (m[1] == -CUDART_INF_F && mx[1] > m[1]);
    if (__any_sync(0xffffffffu, grow)) {   // the reference moves only when a score is well above it (p <= 2^8 otherwise)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = fmaxf(mx[h], m[h]);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float corr = win_rescale(m[h], top);
        m[h] = top;
        l[h] *= corr;
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          o[j][2 * h] *= corr;
          o[j][2 * h + 1] *= corr;
        }
      }
    }
    uint32_t ph[4], pl[4];   // A operand: (row g8, tokens 2 c4), (g8 + 8, 2 c4), (g8, 2 c4 + 8), (g8 + 8, 2 c4 + 8)
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float ref = m[h] == -CUDART_INF_F ? 0.f : m[h];   // nothing seen yet: every score is -inf
        const float p0 = win_exp2(s[n][2 * h] - ref), p1 = win_exp2(s[n][2 * h + 1] - ref);
        l[h] += p0 + p1;
        const __nv_bfloat162 hi = __floats2bfloat162_rn(p0, p1);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(&hi);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xFFFF0000u));
        ph[2 * n + h] = w;
        pl[2 * n + h] = *reinterpret_cast<const uint32_t*>(&lo);
      }
    asm volatile("cp.async.wait_group %0;" ::"n"(kWmRing - 1) : "memory");
    sync_stream();
    {
      const uint32_t at = ring + ((2 * i + 1) % kWmRing) * W::kPiece + v_row * (D * 2);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t v4[4];
        ldmatrix_x4<true>(at + (((2 * j + v_half) ^ (v_row & 7)) << 4), v4);
        mma_bf16_16816(o[2 * j], pl, v4[0], v4[1]);
        mma_bf16_16816(o[2 * j + 1], pl, v4[2], v4[3]);
        mma_bf16_16816(o[2 * j], ph, v4[0], v4[1]);
        mma_bf16_16816(o[2 * j + 1], ph, v4[2], v4[3]);
      }
    }
    sync_stream();
    request(2 * i + 1 + kWmRing);   // takes the values' place
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();   // the rings are free
  float* o_sm = reinterpret_cast<float*>(wm_smem);                       // [stream][row][D]
  float2* ml_sm = reinterpret_cast<float2*>(wm_smem + W::kMl);           // [stream][row]
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = stream * W::kRows + 16 * tile + g8 + 8 * h;
    if (c4 == 0) ml_sm[r] = make_float2(m[h], l[h]);
    if (16 * tile + g8 + 8 * h < n_rows)
#pragma unroll
      for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(o_sm + r * D + 8 * j + 2 * c4) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
  }
  __syncthreads();
  const bool nan = merge_streams<D, kWinThreads, W::kStreams, W::kRows>(o_sm, ml_sm, n_rows);
  if (nan) {
    window_again<D>(a, b, hk, r0, n_rows, t_begin, t_end, len, o_sm, ml_sm);
  }
  window_finish<D>(a, o_sm, ml_sm, n_rows, row_of, seen);
}

template <int D, int kQTerms, int kTiles>
static int32_t launch_window_mma_as(const WindowArgs& a, int batch, const WindowCut& cut, cudaStream_t stream) {
  static DeviceMemo configured;
  if (configure_for_device(window_mma_kernel<D, kQTerms, kTiles>, WmShape<D, kQTerms, kTiles>::kBytes, configured) == 0) return PQ_ERR_CUDA;
  return launch_window(window_mma_kernel<D, kQTerms, kTiles>, a, batch, cut, WmShape<D, kQTerms, kTiles>::kBytes, stream);
}
template <int D, int kQTerms>
static int32_t launch_window_mma_rows(const WindowArgs& a, int rows, int batch, const WindowCut& cut, cudaStream_t stream) {
  return rows == 16 ? launch_window_mma_as<D, kQTerms, 1>(a, batch, cut, stream) : launch_window_mma_as<D, kQTerms, 4>(a, batch, cut, stream);
}

// Which kernel takes a call, the (query, head) rows of its blocks for `all` rows of a kv head, and the streams of tokens in a block.
static bool window_on_tensor_cores(int d, int kv_dtype) { return kv_dtype == PQ_DTYPE_BF16 && d >= 64; }
struct WindowRows {
  int rows, streams, steps;
  int64_t blocks;
};
static WindowRows window_rows_of(int rows, int streams, int steps, int64_t all) {
  WindowRows r = {rows, streams, steps, (all + rows - 1) / rows};
  return r;
}
static WindowRows window_rows_of_lanes(int d, int kv_dtype, int64_t all) {
  return window_rows_of(all == 1 ? 1 : all == 2 ? 2 : all <= 4 ? 4 : 8, kWinWarps, kv_dtype == PQ_DTYPE_F32 && d >= 64 ? d / 32 : 1, all);
}
// On tensor cores 16 rows and four streams are as fast as 64 and one (the blocks that share a window's tokens find them in L2), or faster where
// that leaves no rows empty and needs no parts: 35 rows over 2048 tokens 23.0 and 24.5 us (clusters of four), 32 over 2000 15.3 and 17.3 (32 rows and two
// streams), 64 over 4000 25.4 and 31.6, 64 over 2048 of 32 sequences 132 both.  With more than 48 rows over windows larger than L2 (126 MB) one
// reading is: eight sequences of 8192 138 and 115.
static WindowRows window_rows(int d, int kv_dtype, int batch, int n_q, int n_kv_heads, int g, int max_len) {
  const int64_t all = (int64_t)n_q * g;
  if (!window_on_tensor_cores(d, kv_dtype)) return window_rows_of_lanes(d, kv_dtype, all);
  const bool once = all > 48 && (double)batch * n_kv_heads * max_len * (4 * d) > 126e6;
  return once ? window_rows_of(64, 1, 1, all) : window_rows_of(16, kWinWarps, 1, all);
}
// Parts that a call may leave: of either way to take the rows, so that a smaller bound on the length never needs more.
static int window_most_parts(int d, int batch, int n_q, int n_kv_heads, int g, int max_len) {
  const int64_t all = (int64_t)n_q * g, heads = (int64_t)batch * n_kv_heads;
  int parts = 1;
  for (const WindowRows& r : {window_rows_of_lanes(d, PQ_DTYPE_F32, all), window_rows_of_lanes(d, PQ_DTYPE_BF16, all), window_rows_of(16, kWinWarps, 1, all),
                              window_rows_of(64, 1, 1, all)})
    parts = std::max(parts, cut_window(heads * r.blocks, max_len, kFastMaxGridHost, r.streams, r.steps).parts);
  return parts;
}
static int32_t launch_window_attention(const WindowArgs& a, int kv_dtype, int rows, int batch, const WindowCut& cut, cudaStream_t stream) {
  const bool exact = a.io_dtype == PQ_DTYPE_BF16;   // queries that are one bf16 term
  if (window_on_tensor_cores(a.d, kv_dtype)) {
    if (a.d == 64) return exact ? launch_window_mma_rows<64, 1>(a, rows, batch, cut, stream) : launch_window_mma_rows<64, 3>(a, rows, batch, cut, stream);
    return exact ? launch_window_mma_rows<128, 1>(a, rows, batch, cut, stream) : launch_window_mma_rows<128, 3>(a, rows, batch, cut, stream);
  }
  if (kv_dtype == PQ_DTYPE_BF16)
    return a.d == 16 ? launch_window_rows<__nv_bfloat16, 16>(a, rows, batch, cut, stream) : launch_window_rows<__nv_bfloat16, 32>(a, rows, batch, cut, stream);
  switch (a.d) {
    case 16: return launch_window_rows<float, 16>(a, rows, batch, cut, stream);
    case 32: return launch_window_rows<float, 32>(a, rows, batch, cut, stream);
    case 64: return launch_window_rows<float, 64>(a, rows, batch, cut, stream);
    default: return launch_window_rows<float, 128>(a, rows, batch, cut, stream);
  }
}

// An attention over a window with its arguments checked, and its launch: its parts, where there are several, lie at a.part_out.
struct WindowCall {
  WindowArgs a;
  WindowRows rows;
  int kv_dtype, batch, max_len;
};
static int32_t launch_window_call(const WindowCall& w, bool early, cudaStream_t stream) {
  static DeviceMemo sm_count;
  const int n_sm = sm_count_of_device(sm_count);
  if (n_sm == 0) return PQ_ERR_CUDA;
  WindowArgs a = w.a;
  const WindowCut cut = cut_window((int64_t)w.batch * a.n_kv_heads * w.rows.blocks, w.max_len, std::min(n_sm, kFastMaxGridHost), w.rows.streams,
                                   w.rows.steps);
  a.early = early;
  a.n_parts = cut.parts;
  a.n_splits = cut.cluster * cut.parts;
  a.part_lse = a.part_out + (cut.parts > 1 ? cut.parts * a.n_rows * a.d : 0);
  const int32_t st = launch_window_attention(a, w.kv_dtype, w.rows.rows, w.batch, cut, stream);
  if (st != PQ_OK || cut.parts == 1) return st;
  // the window kernel has reported the rows that see nothing
  return launch_merge(a.d, a.n_rows, cut.parts, a.part_out, PQ_DTYPE_F32, a.part_lse, a.out, a.out_dtype, a.lse, nullptr, stream);
}

}  // namespace pq
