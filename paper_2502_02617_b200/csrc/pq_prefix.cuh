// Attention of many queries over one compressed sequence that all of them see (a shared prefix): the kernel for head_dims below 128, and
// the rotations before and after it and prefix_tc_kernel (included by pq_decode.cu).
//
// prefix_mma_kernel: a block of eight warps takes 16 kTiles rows of a kv head and a range of the tokens.  kTiles warps share a
// stream of tiles of 16 kTiles tokens; 8 / kTiles streams share the range.  Each warp of a stream decodes 16 tokens of a tile
// (DeQuant of Algorithm 1 in float32, a lane half of a token's blocks), the keys as fp16 value and residual (22 bits) and the
// values as fp16, into the stream's piece of shared memory, 16-byte chunks swizzled by the token; then each warp multiplies its
// 16 rows with all tokens of the tile (mma.sync): S = Q'lo K_hi + Q'hi K_lo + Q'hi K_hi with the queries rotated, scaled and split
// the same way before, and O += P V with weights of fp16, whose sum is taken of what the product sees.  The packed codes of a
// stream's next tile are in registers while the present one is decoded and multiplied.  A level's table is at most 16 pairs of
// (cos, sin), 128 bytes: lookups are free of bank conflicts without copies, but two wavefronts each, and shared memory bounds
// the kernel (34 wavefronts per token and kv head at head_dim 128, where the kernels with larger, replicated tables are faster: 16 rows
// over 32768 tokens 57 us against 49).  The streams meet in shared memory, the blocks of a cluster in each other's, and the parts beyond
// that in prefix_unrotate_kernel.
// Measured, 16/8 heads of 64: 16 queries over 4096 tokens 19 us, 64 over 8192 59 (a decode per query took 36 us for the former).
#pragma once

namespace pq {

constexpr int kPxThreads = 256, kPxWarps = kPxThreads / 32, kPxMaxParts = 32;
// Weights are fp16 numbers 2^(s - reference), and a shared prefix is long: a reference at the largest score would leave all below 2^-25 of it at
// 0, and 2^18 tokens at 2^-25.5 are half a percent of the sum.  It is kPxBelow under the largest score of its tile and moves when one is more
// than kPxMost above it, so a weight is 2^15 at most and rounded by 2^-11 of itself or by 2^-32 of the largest one, whichever is more.
// (prefix_mma_kernel's denominator sums the rounded weights, prefix_tc_kernel's the weights before that, which is 2.5 % faster there; the output
// is off by those roundings, N 2^-32 for N small weights, either way.)
constexpr float kPxBelow = 7.f, kPxMost = 15.f;
template <int D, int kTiles>
struct PxShape {
  static constexpr int kStreams = kPxWarps / kTiles, kRows = 16 * kTiles, kT = 16 * kTiles;   // tokens of a stream's tile
  static constexpr int kPiece = kT * D * 2;                           // keys' values, keys' residuals, values: one each
  static constexpr int kOut = kStreams * kRows * D * 4;               // the streams' outputs, where the pieces were
  static constexpr int kArea = 3 * kStreams * kPiece > kOut ? 3 * kStreams * kPiece : kOut;
  static constexpr int kMl = kArea, kTab = kMl + kStreams * kRows * 8;
  static constexpr int kQ = kTab + 256, kBytes = kQ + kTiles * 2 * (D / 16) * 512;
};

struct PrefixKernelArgs {
  int n_q_heads, n_kv_heads, n_queries, n_splits;   // n_splits: see WindowArgs
  int64_t n_rows;
  const Tables* tables;
  const uint8_t* cache;
  const int32_t* len;
  const __half* qrot;    // [row][value | residual][D], coordinate j at (j & ~3) | (0, 2, 1, 3)[j & 3]
  float *part_out, *part_lse;   // [part][row][D] in the rotated basis, [part][row] (natural log)
  int32_t* status;
  Paging pg;
};

// The packed codes of half a token: kBl blocks.
template <int D>
struct PxCodes {
  static constexpr int kBl = D >= 32 ? D / 32 : 1;
  uint32_t l1[kBl], l2, l3, l4, r[(kBl + 1) / 2];
};
template <int D>
__device__ __forceinline__ void px_load(PxCodes<D>& c, const uint8_t* tb, int tok, int half) {
  constexpr int kNb = D / 16, kB1 = 4 * kNb, kB2 = kNb, kB3 = kNb >= 2 ? kNb / 2 : 1, kB4 = kNb >= 4 ? kNb / 4 : 1, kBr = 2 * kNb;
  constexpr int o2 = kTokenBlock * kB1, o3 = o2 + kTokenBlock * kB2, o4 = o3 + kTokenBlock * kB3, orad = o4 + kTokenBlock * kB4;
  const uint8_t *p1 = tb + tok * kB1, *p2 = tb + o2 + tok * kB2, *p3 = tb + o3 + tok * kB3, *p4 = tb + o4 + tok * kB4, *pr = tb + orad + tok * kBr;
  if constexpr (D == 64) {
    const uint2 w = *reinterpret_cast<const uint2*>(p1 + 8 * half);
    c.l1[0] = w.x; c.l1[1] = w.y;
    c.l2 = *reinterpret_cast<const uint16_t*>(p2 + 2 * half);
    c.l3 = p3[half];
    c.l4 = p4[0] >> (4 * half);
    c.r[0] = *reinterpret_cast<const uint32_t*>(pr + 4 * half);
  } else if constexpr (D == 32) {
    c.l1[0] = *reinterpret_cast<const uint32_t*>(p1 + 4 * half);
    c.l2 = p2[half];
    c.l3 = p3[0] >> (4 * half);
    c.l4 = p4[0] >> (2 * half);
    c.r[0] = *reinterpret_cast<const uint16_t*>(pr + 2 * half);
  } else {
    c.l1[0] = *reinterpret_cast<const uint32_t*>(p1);
    c.l2 = p2[0];
    c.l3 = p3[0];
    c.l4 = p4[0];
    c.r[0] = *reinterpret_cast<const uint16_t*>(pr);
  }
}
// DeQuant of block i (without the final S^T), `live`: the token exists.
template <int D>
__device__ __forceinline__ void px_decode(const PxCodes<D>& c, int i, bool live, const uint8_t* tab, float* y) {
  auto entry = [&](int first, uint32_t byte) { return *reinterpret_cast<const float2*>(tab + 8 * first + byte); };   // byte: 8 times the code
  const uint32_t bits = (c.r[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
  const float r = live ? __half2float(__ushort_as_half((unsigned short)bits)) : 0.f;   // stale bytes past the end must not reach the products
  const uint32_t l2 = c.l2 >> (8 * i), l3 = c.l3 >> (4 * i), l4 = c.l4 >> (2 * i);
  const float2 e4 = entry(24, (l4 & 3u) << 3);
  const float r3[2] = {r * e4.x, r * e4.y};
  float r2[4], r1[8];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float2 e = entry(20, (j == 0 ? l3 << 3 : l3 << 1) & 24u);
    r2[2 * j] = r3[j] * e.x;
    r2[2 * j + 1] = r3[j] * e.y;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 e = entry(16, (j == 0 ? l2 << 3 : j == 1 ? l2 << 1 : l2 >> (2 * j - 3)) & 24u);
    r1[2 * j] = r2[j] * e.x;
    r1[2 * j + 1] = r2[j] * e.y;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 e = entry(0, (j == 0 ? c.l1[i] << 3 : c.l1[i] >> (4 * j - 3)) & 120u);
    y[2 * j] = r1[j] * e.x;
    y[2 * j + 1] = r1[j] * e.y;
  }
}
// a - the low half of h, b - the high half, as fp16
__device__ __forceinline__ uint32_t px_residual(float a, float b, uint32_t h) {
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "mov.b32 {lo, hi}, %2;\n\t"
      "add.rn.f32.f16 %0, lo, %0;\n\t"
      "add.rn.f32.f16 %1, hi, %1;\n\t}"
      : "+f"(a), "+f"(b)
      : "r"(h ^ 0x80008000u));
  return as_u32(__floats2half2_rn(a, b));
}

template <int D, int kTiles>
__global__ void __launch_bounds__(kPxThreads, kTiles <= 2 ? 2 : 1) prefix_mma_kernel(const __grid_constant__ PrefixKernelArgs a) {
  using W = PxShape<D, kTiles>;
  constexpr int kSteps = D / 16, kT = W::kT, kThreads = 32 * kTiles, kBl = PxCodes<D>::kBl, kN = 2 * kTiles;   // kN: groups of eight tokens of a tile
  constexpr int kCh = D / 8 < 8 ? D / 8 : 8, kSh = kCh == 8 ? 0 : kCh == 4 ? 1 : 2;   // chunk x of token t lies at x ^ swizzle(t)
  extern __shared__ __align__(128) uint8_t px_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, c4 = lane & 3;
  const int stream = warp / kTiles, tile = warp % kTiles;
  const int g = a.n_q_heads / a.n_kv_heads, hk = blockIdx.y, n_splits = a.n_splits, rb = blockIdx.x / n_splits, split = blockIdx.x % n_splits;
  const int r0 = rb * W::kRows, n_rows = min(W::kRows, a.n_queries * g - r0);   // row r0 + r: query (r0 + r) / g, head hk * g + (r0 + r) % g
  const uint32_t sm = (uint32_t)__cvta_generic_to_shared(px_smem);
  if (tid < PQ_N_CENTROIDS) reinterpret_cast<float2*>(px_smem + W::kTab)[tid] = make_float2(a.tables->cen_cos[tid], a.tables->cen_sin[tid]);   // a constant
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // behind the wait: see WindowArgs::early
  const int len = max(*a.len, 0);
  const int tiles_all = (len + kT - 1) / kT;
  const int first = (int)((int64_t)tiles_all * split / n_splits), n_tiles = (int)((int64_t)tiles_all * (split + 1) / n_splits) - first;
  const int mine = n_tiles > stream ? (n_tiles - stream + W::kStreams - 1) / W::kStreams : 0;
  auto row_of = [&](int r) -> int64_t {
    const int j = (r0 + r) / g;
    return (int64_t)j * a.n_q_heads + hk * g + (r0 + r - j * g);
  };
  // ---- packed codes: lane = (token, half of its blocks) of the warp's 16 tokens of a tile
  const Layout L = make_layout(D, a.pg.page_tokens);
  const int tok = lane & 15, half = lane >> 4;
  PxCodes<D> kc, vc;
  auto request = [&](int i) {
    const int t0 = (first + stream + i * W::kStreams) * kT + 16 * tile;
    const uint8_t* tb = a.cache + kv_block_pair_offset(L, a.pg, a.n_kv_heads, 0, hk, t0 / kTokenBlock, a.status);
    px_load<D>(kc, tb, t0 % kTokenBlock + tok, half);
    px_load<D>(vc, tb + L.block_bytes, t0 % kTokenBlock + tok, half);
  };
  if (mine > 0) request(0);
  // ---- queries: A operand of rows g8 and g8 + 8 of the warp's tile (rows past the last repeat it); the streams share the work
  uint4* q_sm = reinterpret_cast<uint4*>(px_smem + W::kQ) + tile * (2 * kSteps * 32) + lane;
  {
    const __half* lo = a.qrot + row_of(min(16 * tile + g8, n_rows - 1)) * (2 * D) + 2 * c4;
    const __half* hi = a.qrot + row_of(min(16 * tile + g8 + 8, n_rows - 1)) * (2 * D) + 2 * c4;
    for (int i = stream; i < 2 * kSteps; i += W::kStreams)   // value fragments, then residuals
      q_sm[i * 32] = make_uint4(*reinterpret_cast<const uint32_t*>(lo + 16 * i), *reinterpret_cast<const uint32_t*>(hi + 16 * i),
                                *reinterpret_cast<const uint32_t*>(lo + 16 * i + 8), *reinterpret_cast<const uint32_t*>(hi + 16 * i + 8));
  }
  __syncthreads();
  auto sync_stream = [&]() {
    if constexpr (kTiles == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + stream), "n"(kThreads) : "memory");
  };
  const uint32_t piece = sm + stream * (3 * W::kPiece);   // keys' values; residuals and values behind them
  const uint32_t put = piece + (16 * tile + tok) * (D * 2);
  const uint32_t swz = (uint32_t)((tok >> kSh) & (kCh - 1));
  const uint8_t* tab = px_smem + W::kTab;

  float o[D / 8][4], m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};   // of rows g8 and g8 + 8; l: this lane's share
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  const int k_row = (lane & 7) + ((lane >> 4) << 3), k_half = (lane >> 3) & 1;        // ldmatrix of keys: token, 8-coordinate half
  const int v_row = (lane & 7) + (((lane >> 3) & 1) << 3), v_half = lane >> 4;        // of values
  const uint32_t k_swz = (uint32_t)((k_row >> kSh) & (kCh - 1)), v_swz = (uint32_t)((v_row >> kSh) & (kCh - 1));
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    const int t0 = (first + stream + i * W::kStreams) * kT;
    const bool live = t0 + 16 * tile + tok < len;
    if (D >= 32 || half == 0) {
#pragma unroll
      for (int e = 0; e < kBl; ++e) {
        const int blk = half * kBl + e;
        const uint32_t at0 = put + (((2 * blk) ^ swz) << 4), at1 = put + (((2 * blk + 1) ^ swz) << 4);
        float y[16];
        px_decode<D>(kc, e, live, tab, y);
        uint32_t h[8], w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {   // pairs (0, 2), (1, 3) of every four: the order of the queries
          const float p = y[4 * (j >> 1) + (j & 1)], q = y[4 * (j >> 1) + (j & 1) + 2];
          h[j] = as_u32(__floats2half2_rn(p, q));
          w[j] = px_residual(p, q, h[j]);
        }
        pt_sts128(at0, h[0], h[1], h[2], h[3]);
        pt_sts128(at1, h[4], h[5], h[6], h[7]);
        pt_sts128(at0 + W::kPiece, w[0], w[1], w[2], w[3]);
        pt_sts128(at1 + W::kPiece, w[4], w[5], w[6], w[7]);
        px_decode<D>(vc, e, live, tab, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = as_u32(__floats2half2_rn(y[2 * j], y[2 * j + 1]));
        pt_sts128(at0 + 2 * W::kPiece, h[0], h[1], h[2], h[3]);
        pt_sts128(at1 + 2 * W::kPiece, h[4], h[5], h[6], h[7]);
      }
    }
    if (i + 1 < mine) request(i + 1);
    sync_stream();
    float s[kN][4];   // tokens t0 + 8 n + 2 c4, + 1 of rows g8 (0, 1) and g8 + 8 (2, 3)
#pragma unroll
    for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int ks = 0; ks < kSteps; ++ks) {
      const uint4 qh = q_sm[ks * 32], ql = q_sm[(kSteps + ks) * 32];
#pragma unroll
      for (int n2 = 0; n2 < kTiles; ++n2) {
        const uint32_t at = piece + (16 * n2 + k_row) * (D * 2) + (((2 * ks + k_half) ^ k_swz) << 4);
        uint32_t hi[4], lo[4];
        ldmatrix_x4<false>(at, hi);
        ldmatrix_x4<false>(at + W::kPiece, lo);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mma_16816(s[2 * n2 + e], ql.x, ql.y, ql.z, ql.w, hi[2 * e], hi[2 * e + 1]);
          mma_16816(s[2 * n2 + e], qh.x, qh.y, qh.z, qh.w, lo[2 * e], lo[2 * e + 1]);
          mma_16816(s[2 * n2 + e], qh.x, qh.y, qh.z, qh.w, hi[2 * e], hi[2 * e + 1]);
        }
      }
    }
    if (t0 + kT > len) {
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 8 * n + 2 * c4 + (e & 1) >= len) s[n][e] = -CUDART_INF_F;
    }
    float mx[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) mx[h] = fmaxf(mx[h], fmaxf(s[n][2 * h], s[n][2 * h + 1]));
    const bool grow = mx[0] > m[0] + kPxMost || mx[1] > m[1] + kPxMost;   // true on the first tile (m is -inf), which has a token
    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = mx[h];
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = fmaxf(top - kPxBelow, m[h]);
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
    const float ref[2] = {m[0] == -CUDART_INF_F ? 0.f : m[0], m[1] == -CUDART_INF_F ? 0.f : m[1]};   // only scores of -inf so far
#pragma unroll
    for (int n2 = 0; n2 < kTiles; ++n2) {
      uint32_t p[4];   // A operand: (row g8, tokens 2 c4), (g8 + 8, 2 c4), (g8, 2 c4 + 8), (g8 + 8, 2 c4 + 8)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w = as_u32(__floats2half2_rn(fast_exp2(s[2 * n2 + n][2 * h] - ref[h]), fast_exp2(s[2 * n2 + n][2 * h + 1] - ref[h])));
          pt_add_halves(l[h], w);   // the denominator of what the product sees
          p[2 * n + h] = w;
        }
      const uint32_t at = piece + 2 * W::kPiece + (16 * n2 + v_row) * (D * 2);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t v4[4];
        ldmatrix_x4<true>(at + (((2 * j + v_half) ^ v_swz) << 4), v4);
        mma_16816(o[2 * j], p[0], p[1], p[2], p[3], v4[0], v4[1]);
        mma_16816(o[2 * j + 1], p[0], p[1], p[2], p[3], v4[2], v4[3]);
      }
    }
    sync_stream();   // the pieces may be written again
  }
  __syncthreads();
  float* o_sm = reinterpret_cast<float*>(px_smem);                       // [stream][row][D]
  float2* ml_sm = reinterpret_cast<float2*>(px_smem + W::kMl);           // [stream][row]
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
  merge_streams<D, kPxThreads, W::kStreams, W::kRows>(o_sm, ml_sm, n_rows);
  uint32_t n_blocks;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(n_blocks));
  const int64_t part = split / n_blocks;
  cluster_merge<D, kPxThreads>(o_sm, ml_sm, n_rows, [&](int r, int c, const float4& acc, float lse) {
    const int64_t row = row_of(r);
    *reinterpret_cast<float4*>(a.part_out + (part * a.n_rows + row) * D + c) = acc;
    if (c == 0) a.part_lse[part * a.n_rows + row] = lse;
  });
}

// ---- the rotations before and after, on tensor cores (mma.sync)
// A block of eight warps takes 16 rows (32 and 64 at head_dim 32 and 16); a warp has kNt columns of eight.  S is copied to shared memory
// before the kernel ahead in the stream has finished.  Before the attention its elements and float32 queries are three bf16 terms each (24 bits,
// so that the scores keep the 22 of the rotated queries and keys; two moved the log-sum-exp of scores of a few hundred by twice as much as the
// rest), bf16 queries are one.  After it two of each are enough: an error of 2^-16 on outputs whose values carry 2^-12.  Small products first.
template <int D>
struct PrShape {
  static constexpr int kNt = D == 128 ? 2 : 1, kTileWarps = D / 8 / kNt, kTiles = 8 / kTileWarps, kRows = 16 * kTiles, kSteps = D / 16;
  static constexpr int kStride = D + 4, kXStride = D + 8;   // floats of a row of S: four lanes' rows lie in different banks; of a row of x
  static constexpr int kBytes = (D * kStride + kRows * kXStride + kRows) * 4;
};
constexpr int kPrThreads = 256;
template <int kTerms>
__device__ __forceinline__ void pr_terms(float a, float b, uint32_t* t) {
#pragma unroll
  for (int i = 0; i < kTerms; ++i) {
    const __nv_bfloat162 w = __floats2bfloat162_rn(a, b);
    t[i] = *reinterpret_cast<const uint32_t*>(&w);
    a -= __uint_as_float(t[i] << 16);
    b -= __uint_as_float(t[i] & 0xFFFF0000u);
  }
}
template <int D>
__device__ __forceinline__ void pr_stage(const float* S, float* s) {
#pragma unroll 8
  for (int i = threadIdx.x; i < D * D / 4; i += kPrThreads)
    *reinterpret_cast<float4*>(s + i / (D / 4) * PrShape<D>::kStride + 4 * (i % (D / 4))) = __ldg(reinterpret_cast<const float4*>(S) + i);
}
// d += a times columns n .. n + 7 of S (kTransposed: of S^T) at k-step ks; kTerms: of a, kOfS: of S.
template <int D, bool kTransposed, int kTerms, int kOfS>
__device__ __forceinline__ void pr_mma(float* d, const uint32_t (&a)[kTerms][4], const float* s, int ks, int n, int g8, int c4) {
  constexpr int kStride = PrShape<D>::kStride;
  uint32_t f[2][kOfS];
#pragma unroll
  for (int e = 0; e < 2; ++e) {   // rows 2 c4, + 1 of the step's first or second eight, column n + g8
    const int k = 16 * ks + 8 * e + 2 * c4;
    float2 v;
    if constexpr (kTransposed) v = *reinterpret_cast<const float2*>(s + (n + g8) * kStride + k);
    else v = make_float2(s[k * kStride + n + g8], s[(k + 1) * kStride + n + g8]);
    pr_terms<kOfS>(v.x, v.y, f[e]);
  }
#pragma unroll
  for (int order = kOfS - 1; order >= 0; --order)   // products below 2^(-8 kOfS) are left out
#pragma unroll
    for (int i = kTerms - 1; i >= 0; --i)
      if (i <= order) mma_bf16_16816(d, a[i], f[0][order - i], f[1][order - i]);
}

// q' = (q S) * factor of every row as fp16 value and residual: qrot [row][value | residual][D], coordinate j at (j & ~3) | (0, 2, 1, 3)[j & 3].
template <int D, bool kBf16>
__global__ void __launch_bounds__(kPrThreads) prefix_rotate_kernel(const float* S, const void* q, int64_t n_rows, float factor, __half* qrot) {
  using W = PrShape<D>;
  extern __shared__ __align__(16) float pr_smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, c4 = lane & 3;
  const int64_t row0 = (int64_t)blockIdx.x * W::kRows + 16 * (warp / W::kTileWarps);
  const int n0 = 8 * W::kNt * (warp % W::kTileWarps);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  pr_stage<D>(S, pr_smem);   // a constant of the caller
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t at[2] = {min(row0 + g8, n_rows - 1) * D + 2 * c4, min(row0 + g8 + 8, n_rows - 1) * D + 2 * c4};   // rows past the last repeat it
  constexpr int kTerms = kBf16 ? 1 : 3;
  uint32_t a[W::kSteps][kTerms][4];
#pragma unroll
  for (int ks = 0; ks < W::kSteps; ++ks)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t k = at[i & 1] + 16 * ks + 8 * (i >> 1);
      if constexpr (kBf16) {
        a[ks][0][i] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(q) + k);
      } else {
        const float2 v = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(q) + k);
        uint32_t w[kTerms];
        pr_terms<kTerms>(v.x, v.y, w);
#pragma unroll
        for (int e = 0; e < kTerms; ++e) a[ks][e][i] = w[e];
      }
    }
  __syncthreads();
  float acc[W::kNt][4];
#pragma unroll
  for (int t = 0; t < W::kNt; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
#pragma unroll
  for (int ks = 0; ks < W::kSteps; ++ks)
#pragma unroll
    for (int t = 0; t < W::kNt; ++t) pr_mma<D, false, kTerms, 3>(acc[t], a[ks], pr_smem, ks, n0 + 8 * t, g8, c4);
#pragma unroll
  for (int t = 0; t < W::kNt; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // columns 4 m, 4 m + 1 of the even lane and 4 m + 2, 4 m + 3 of the odd one: the even lane stores the first of each, the odd one the second
      const float mine0 = acc[t][2 * h] * factor, mine1 = acc[t][2 * h + 1] * factor;
      const float other = __shfl_xor_sync(0xffffffffu, c4 & 1 ? mine0 : mine1, 1);
      const float x = c4 & 1 ? other : mine0, y = c4 & 1 ? mine1 : other;
      const __half2 hi = __floats2half2_rn(x, y);
      const __half2 lo = __floats2half2_rn(x - __low2float(hi), y - __high2float(hi));
      const int64_t row = row0 + g8 + 8 * h;
      if (row < n_rows) {
        __half* to = qrot + row * 2 * D + n0 + 8 * t + 4 * (c4 >> 1) + 2 * (c4 & 1);
        *reinterpret_cast<__half2*>(to) = hi;
        *reinterpret_cast<__half2*>(to + D) = lo;
      }
    }
}

// out = (sum_p w_p part_p) S^T + w tail with weights exp(lse - total): parts [part][row][D] in the rotated basis, lse [part][row]
// (natural log; -inf: nothing seen), and, if not null, another partial result tail [row][D], tail_lse [row] in the original
// basis.  n_parts at most kPxMaxParts.
template <int D>
__global__ void __launch_bounds__(kPrThreads) prefix_unrotate_kernel(const float* S, const float* parts, const float* lse, int n_parts, const float* tail,
                                                                     const float* tail_lse, int64_t n_rows, void* out, int out_dtype, float* lse_out,
                                                                     int32_t* status) {
  using W = PrShape<D>;
  constexpr int kV = D >= 64 ? 4 : 2, kRowLanes = D / kV;   // a row's lanes
  extern __shared__ __align__(16) float pr_smem[];
  float* x = pr_smem + D * W::kStride;          // the merged rows
  float* tail_w = x + W::kRows * W::kXStride;   // the tail's weights
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g8 = lane >> 2, c4 = lane & 3;
  const int64_t row0 = (int64_t)blockIdx.x * W::kRows;
  const int tile = warp / W::kTileWarps, n0 = 8 * W::kNt * (warp % W::kTileWarps);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  pr_stage<D>(S, pr_smem);   // a constant of the caller
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the parts come from the kernels before this one
  // a warp merges kMine rows, all of them at a time
  constexpr int kMine = W::kRows / 8, kAtOnce = kMine < 2 ? kMine : 2;
  const int col = lane < kRowLanes ? kV * lane : 0;
#pragma unroll 1
  for (int i0 = 0; i0 < kMine; i0 += kAtOnce) {
    float acc[kAtOnce][kV], w_mine[kAtOnce], mx[kAtOnce], other[kAtOnce];
    int64_t row[kAtOnce];
    bool seen[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {   // rows past the last repeat it
      row[i] = min(row0 + warp + 8 * (i0 + i), n_rows - 1);
      w_mine[i] = lane < n_parts ? lse[lane * n_rows + row[i]] : -CUDART_INF_F;
      other[i] = tail != nullptr ? tail_lse[row[i]] : -CUDART_INF_F;
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      mx[i] = fmaxf(w_mine[i], other[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], o));
      seen[i] = mx[i] > -CUDART_INF_F || __any_sync(0xffffffffu, w_mine[i] != w_mine[i] || other[i] != other[i]);   // a NaN part makes the row NaN
      w_mine[i] = w_mine[i] == -CUDART_INF_F ? 0.f : __expf(w_mine[i] - mx[i]);
#pragma unroll
      for (int e = 0; e < kV; ++e) acc[i][e] = 0.f;
    }
#pragma unroll 4
    for (int p = 0; p < n_parts; ++p) {   // part order
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float w = __shfl_sync(0xffffffffu, w_mine[i], p);
        const float* src = parts + (p * n_rows + row[i]) * D + col;
        if constexpr (kV == 4) {
          const float4 v = *reinterpret_cast<const float4*>(src);
          acc[i][0] = fmaf(w, v.x, acc[i][0]);
          acc[i][1] = fmaf(w, v.y, acc[i][1]);
          acc[i][2 % kV] = fmaf(w, v.z, acc[i][2 % kV]);
          acc[i][3 % kV] = fmaf(w, v.w, acc[i][3 % kV]);
        } else {
          const float2 v = *reinterpret_cast<const float2*>(src);
          acc[i][0] = fmaf(w, v.x, acc[i][0]);
          acc[i][1] = fmaf(w, v.y, acc[i][1]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int r = warp + 8 * (i0 + i);
      float sum = w_mine[i];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      const float w_other = other[i] == -CUDART_INF_F ? 0.f : __expf(other[i] - mx[i]);
      sum += w_other;
      const float inv = seen[i] ? 1.f / sum : 0.f;   // a query that sees no token: zeros (its parts hold zeros)
      if (lane == 0) {
        tail_w[r] = w_other == 0.f ? 0.f : w_other * inv;   // not 0 times a NaN
        if (row0 + r < n_rows) {
          if (lse_out != nullptr) lse_out[row[i]] = seen[i] ? mx[i] + __logf(sum) : -CUDART_INF_F;
          else if (!seen[i]) set_status(status, PQ_ERR_EMPTY);
        }
      }
      if (lane < kRowLanes)
#pragma unroll
        for (int e = 0; e < kV; e += 2) *reinterpret_cast<float2*>(x + r * W::kXStride + kV * lane + e) = make_float2(acc[i][e] * inv, acc[i][e + 1] * inv);
    }
  }
  __syncthreads();
  float y[W::kNt][4];
#pragma unroll
  for (int t = 0; t < W::kNt; ++t) y[t][0] = y[t][1] = y[t][2] = y[t][3] = 0.f;
#pragma unroll
  for (int ks = 0; ks < W::kSteps; ++ks) {
    uint32_t a[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = *reinterpret_cast<const float2*>(x + (16 * tile + g8 + 8 * (i & 1)) * W::kXStride + 16 * ks + 2 * c4 + 8 * (i >> 1));
      uint32_t w[2];
      pr_terms<2>(v.x, v.y, w);
      a[0][i] = w[0];
      a[1][i] = w[1];
    }
#pragma unroll
    for (int t = 0; t < W::kNt; ++t) pr_mma<D, true, 2, 2>(y[t], a, pr_smem, ks, n0 + 8 * t, g8, c4);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = 16 * tile + g8 + 8 * h;
    const int64_t row = row0 + r;
    if (row >= n_rows) continue;
    const float w = tail_w[r];
#pragma unroll
    for (int t = 0; t < W::kNt; ++t) {
      const int64_t at = row * D + n0 + 8 * t + 2 * c4;
      float v0 = y[t][2 * h], v1 = y[t][2 * h + 1];
      if (tail != nullptr && w != 0.f) {   // a part without tokens may hold anything
        const float2 v = *reinterpret_cast<const float2*>(tail + at);
        v0 = fmaf(w, v.x, v0);
        v1 = fmaf(w, v.y, v1);
      }
      if (out_dtype == PQ_DTYPE_BF16) *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = __floats2bfloat162_rn(v0, v1);
      else *reinterpret_cast<float2*>(reinterpret_cast<float*>(out) + at) = make_float2(v0, v1);
    }
  }
}
template <int D>
static int32_t launch_prefix_rotate(const float* S, const void* q, int io_dtype, int64_t n_rows, float factor, __half* qrot, cudaStream_t stream) {
  const dim3 grid((unsigned)((n_rows + PrShape<D>::kRows - 1) / PrShape<D>::kRows));
  static DeviceMemo configured[2];
  void (*kernel)(const float*, const void*, int64_t, float, __half*) = io_dtype == PQ_DTYPE_BF16 ? prefix_rotate_kernel<D, true> : prefix_rotate_kernel<D, false>;
  if (configure_for_device(kernel, PrShape<D>::kBytes, configured[io_dtype == PQ_DTYPE_BF16]) == 0) return PQ_ERR_CUDA;
  return launch_dependent(kernel, grid, kPrThreads, PrShape<D>::kBytes, stream, S, q, n_rows, factor, qrot);
}
template <int D>
static int32_t launch_prefix_unrotate(const float* S, const float* parts, const float* lse, int n_parts, const float* tail, const float* tail_lse,
                                      int64_t n_rows, void* out, int out_dtype, float* lse_out, int32_t* status, cudaStream_t stream) {
  const dim3 grid((unsigned)((n_rows + PrShape<D>::kRows - 1) / PrShape<D>::kRows));
  static DeviceMemo configured;
  if (configure_for_device(prefix_unrotate_kernel<D>, PrShape<D>::kBytes, configured) == 0) return PQ_ERR_CUDA;
  return launch_dependent(prefix_unrotate_kernel<D>, grid, kPrThreads, PrShape<D>::kBytes, stream, S, parts, lse, n_parts, tail, tail_lse, n_rows, out, out_dtype, lse_out,
                          status);
}

// How a call is cut: row tiles of a block, row blocks, blocks of a cluster, parts.
struct PrefixCut {
  int tiles, row_blocks, cluster, parts;
};
static PrefixCut cut_prefix(int n_queries, int n_kv_heads, int g, int max_len, int n_sm) {
  const int64_t all = (int64_t)n_queries * g;
  PrefixCut c;
  c.tiles = all <= 16 ? 1 : all <= 32 ? 2 : 4;
  c.row_blocks = (int)((all + 16 * c.tiles - 1) / (16 * c.tiles));
  const int64_t units = (int64_t)n_kv_heads * c.row_blocks, room = (c.tiles <= 2 ? 2 : 1) * (int64_t)n_sm;
  const int64_t tokens = 16 * kPxWarps, most = ((int64_t)max_len + tokens - 1) / tokens;   // a tile for every stream of a block
  const int64_t splits = std::max<int64_t>(1, std::min(room / units, most));
  c.cluster = 1;
  while (c.cluster < kWinMaxCluster && 2 * c.cluster <= splits) c.cluster *= 2;
  c.parts = c.cluster == kWinMaxCluster ? (int)std::min<int64_t>(kPxMaxParts, splits / kWinMaxCluster) : 1;
  return c;
}
// The workspace: rotated queries, parts, their log-sum-exps.
static int64_t prefix_workspace_bytes(int d, int64_t n_rows, int64_t parts) { return n_rows * 4 * d + parts * n_rows * (d + 1) * 4; }

template <int D, int kTiles>
static int32_t launch_prefix_mma(const PrefixKernelArgs& a, const PrefixCut& cut, cudaStream_t stream) {
  static DeviceMemo configured;
  if (configure_for_device(prefix_mma_kernel<D, kTiles>, PxShape<D, kTiles>::kBytes, configured) == 0) return PQ_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.n_splits * cut.row_blocks, a.n_kv_heads);
  cfg.blockDim = dim3(kPxThreads);
  cfg.dynamicSmemBytes = PxShape<D, kTiles>::kBytes;
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, prefix_mma_kernel<D, kTiles>, a);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    cudaGetLastError();
    return PQ_ERR_CUDA;
  }
  return launch_status();
}
// What an attention over a shared prefix writes: out and lse, or, with a window, the attention over both to `out` alone.
struct SharedPrefix {
  void* out;
  int out_dtype;
  float* lse;
  const WindowCall* window;     // the window that follows the prefix (pq_shared_attention); may be null
  float *part_out, *part_lse;   // with a window: room for the prefix's own result, where a kernel rotates back by itself
};
// The end of a call whose kernel has left `n_parts` parts in the rotated basis.
template <int D>
static int32_t finish_prefix(const DecodeArgs& d, const SharedPrefix& shared, const float* parts, const float* lse, int n_parts, cudaStream_t stream) {
  const int64_t n_rows = (int64_t)d.n_q * d.n_q_heads;
  const float *tail = nullptr, *tail_lse = nullptr;
  if (shared.window != nullptr) {
    const int32_t st = launch_window_call(*shared.window, true, stream);
    if (st != PQ_OK) return st;
    tail = reinterpret_cast<const float*>(shared.window->a.out);
    tail_lse = shared.window->a.lse;
  }
  return launch_prefix_unrotate<D>(d.S, parts, lse, n_parts, tail, tail_lse, n_rows, shared.out, shared.out_dtype, shared.lse, d.status, stream);
}
template <int D>
static int32_t launch_prefix(const DecodeArgs& d, const SharedPrefix& shared, void* workspace, const PrefixCut& cut, cudaStream_t stream) {
  PrefixKernelArgs a;
  a.n_q_heads = d.n_q_heads; a.n_kv_heads = d.n_kv_heads; a.n_queries = d.n_q; a.n_splits = cut.cluster * cut.parts;
  a.n_rows = (int64_t)d.n_q * d.n_q_heads;
  a.tables = d.tables; a.cache = d.cache; a.len = d.lens; a.status = d.status; a.pg = d.pg;
  __half* qrot = reinterpret_cast<__half*>(workspace);
  a.qrot = qrot;
  a.part_out = reinterpret_cast<float*>(qrot + a.n_rows * 2 * D);
  a.part_lse = a.part_out + cut.parts * a.n_rows * D;
  const float factor = d.scale * 1.4426950408889634f;
  int32_t st = launch_prefix_rotate<D>(d.S, d.q, d.io_dtype, a.n_rows, factor, qrot, stream);
  if (st != PQ_OK) return st;
  st = cut.tiles == 1 ? launch_prefix_mma<D, 1>(a, cut, stream) : cut.tiles == 2 ? launch_prefix_mma<D, 2>(a, cut, stream) : launch_prefix_mma<D, 4>(a, cut, stream);
  if (st != PQ_OK) return st;
  return finish_prefix<D>(d, shared, a.part_out, a.part_lse, cut.parts, stream);
}

}  // namespace pq
