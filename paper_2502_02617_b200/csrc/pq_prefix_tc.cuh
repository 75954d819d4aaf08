// Attention of many queries over one compressed sequence that all of them see, head_dim 128, on the 5th-generation tensor cores
// (included by pq_decode.cu): the roles and operands of prefill_tc_kernel, without a causal limit, with twice the row owners and a
// third more decoders.
//
// A CTA of 24 warps owns 128 (query, head) rows of a kv head, two CTAs share one 256-row MMA (cta_group::2) and loop over a range of the
// 64-token blocks, each decoding half of a block.
//   * warp 22 requests the packed blocks, four in flight; with a decoder warp that asks for them between its pieces a block came 7 % later
//   * warps 8-21 (decoders) DeQuant the packed blocks into swizzled tiles: keys as fp16 value and residual, values as fp16;
//   * warp 23 issues S = Q'lo K_hi^T + Q'hi K_lo^T + Q'hi K_hi^T into one of four score accumulators and O += P V_hat;
//   * warps 0-7 (row owners): thread = row and half of a block's tokens.  A row's two threads exchange their maxima through shared memory
//     and one barrier of the eight warps, take the same lazy reference, and write 16 columns of P each.  80 registers a thread
//     are enough for half a row, so that 24 warps fit where 16 do with a whole row.
// Bound by instruction issue and the latency of the lookups: 0.93 us per block of a pair at first (prefill_tc_kernel 1.0) with 4900 warp
// instructions per CTA, now about 4000; then, without the lookups 0.84, without the exponentials 0.82, without both 0.69, and with a third of the
// score MMAs as well 0.62.  A CTA alone with 128 rows, whole blocks and two stages takes 1.5 us a block and is faster nowhere.  Measured with the
// rotations, 32/8 heads: 64 queries over 32768 tokens 75 us (90 in prefill_tc_kernel); the kernel alone 71 with caches cold, its MMAs 56 % of that.
#pragma once

#include "pq_tc_common.cuh"

namespace pq {

constexpr int kPcGroups = 8;   // warp-sized pieces of a block's decoding in a CTA
constexpr int kPcOwners = 8, kPcDecoders = 14, kPcFetchWarp = kPcOwners + kPcDecoders, kPcMmaWarp = kPcFetchWarp + 1, kPcThreads = 32 * (kPcMmaWarp + 1);
constexpr uint32_t kPcMax = (kPtMisc + 16 + 15) / 16 * 16;   // floats [2][2][128], behind that map
constexpr int kPcSmTotal = (int)(kPcMax + 2 * 2 * 128 * 4 - kPtBase);
static_assert(kPcSmTotal <= 227 * 1024, "shared memory of one CTA");

// A barrier of the row owners; true if the wait of any of them has failed.
__device__ __forceinline__ bool pc_owners_failed(bool fail) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.aligned.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)fail), "n"(32 * kPcOwners)
      : "memory");
  return any != 0;
}
__global__ void __launch_bounds__(kPcThreads, 1) prefix_tc_kernel(DecodeArgs a) {
  extern __shared__ __align__(1024) uint8_t pc_smem_raw[];
  uint8_t* smem = pc_smem_raw - kPtBase;
  const uint32_t sb = tc_smem_u32(pc_smem_raw) - kPtBase;   // the window: rank << 24
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // known to be uniform
  const int g = a.n_q_heads / a.n_kv_heads;
  const int qb_rows = kPtRows / g;                      // queries of a CTA
  const int n_q = a.n_q, n_splits = a.n_splits, split = blockIdx.z;   // a pair takes one of n_splits ranges of the blocks
  const int q0 = blockIdx.x * qb_rows, hk = blockIdx.y;
  const int n_rows = max(0, min(qb_rows, n_q - q0)) * g;   // rows in use; row r = (query q0 + r / g, head hk * g + r % g);
                                                           // none in the CTA that only completes a pair
  uint32_t crank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(crank));
  const bool leader = crank == 0;   // the CTA whose thread issues the MMAs and whose barriers collect the arrivals
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kPtMisc + 4);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kPtMisc);
  auto row_index = [&](int r) -> int64_t {               // offset of row r in q / out ([batch][n_q][n_q_heads][128])
    return ((int64_t)(q0 + r / g) * a.n_q_heads + hk * g + r % g) * 128;
  };
  if (sb & 0xFFFFFFu) {   // the host asks for the place (window_as_mapped): never, and then NaN rather than anything (both CTAs leave alike)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int r = tid; r < n_rows; r += kPcThreads) a.part_lse[(int64_t)split * a.batch * a.n_q_heads + row_index(r) / 128] = CUDART_NAN_F;
    set_status(a.status, PQ_ERR_CUDA);
    return;
  }
  if (warp == kPcFetchWarp && lane == 0) {   // this thread uses some of them before the block has met
    for (int i = 0; i < kPtStages; ++i) {
      tc_mbar_init(sb + kPtBarKv + 8 * i, 2 * kPcGroups);    // one arrival per decoded piece (of both CTAs)
      tc_mbar_init(sb + kPtBarPv + 8 * i, 1);                // tcgen05.commit after the value MMA that read the stage
    }
    for (int i = 0; i < kPtRawBufs; ++i) {
      tc_mbar_init(sb + kPtBarRawFull + 8 * i, 1);           // the bytes of a bulk copy
      tc_mbar_init(sb + kPtBarRawEmpty + 8 * i, kPcGroups);  // one arrival per decoded piece
    }
    for (int i = 0; i < kPtScores; ++i) {
      tc_mbar_init(sb + kPtBarS + 8 * i, 1);   // tcgen05.commit
      tc_mbar_init(sb + kPtBarP + 8 * i, 2 * kPcOwners);   // one arrival per row-owner warp (of both CTAs)
    }
    tc_mbar_init(sb + kPtBarDrain, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < 512) build_fast_tables<512>(smem + kPtTab, a.tables);   // from the caller's tables, which no kernel writes (4096 entries)
  if (warp == kPcMmaWarp) {   // the same warp of both CTAs, the same destination offset
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(sb + kPtMisc) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // a programmatic dependent of the kernel before it: its results (lengths, cache, queries) are read only after this wait
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // behind the wait: see WindowArgs::early
  const int len = max(a.lens[0], 0);
  const int all_blocks = (len + kTokenBlock - 1) / kTokenBlock;
  const int jb0 = (int)((int64_t)all_blocks * split / n_splits);                       // this pair's blocks are jb0 + jb,
  const int n_blocks = (int)((int64_t)all_blocks * (split + 1) / n_splits) - jb0;      // 0 <= jb < n_blocks
  const Layout L = make_layout(128, a.pg.page_tokens);
  auto request = [&](int j) {   // packed block j of the range
    const int f = j % kPtRawBufs;
    tc_mbar_expect_tx(sb + kPtBarRawFull + 8 * f, kPtRawBytes);
    bulk_load(sb + kPtRaw + f * kPtRawBytes, a.cache + kv_block_pair_offset(L, a.pg, a.n_kv_heads, 0, hk, jb0 + j, a.status), kPtRawBytes,
              sb + kPtBarRawFull + 8 * f);
  };
  if (warp == kPcFetchWarp && lane == 0)   // the first ones are on their way while the queries are brought in
    for (int j = 0; j < min(kPtRawBufs, n_blocks); ++j) request(j);
  // ---- Q' (fp16 value | residual, rotate_rows_kernel) of this CTA's rows: staged in shared memory with coalesced copies, then
  // written to tensor memory by the row owners (lane = row, two k values per column).  Rows that do not exist repeat the
  // last one (they are not stored).
  for (int i = tid; i < kPtRows * 32; i += kPcThreads) {
    const int r = i >> 5, piece = i & 31;
    const uint32_t dst = sb + kPtKv + r * (2 * kPtQStride * 2) + (piece >> 4) * (kPtQStride * 2) + (piece & 15) * 16;
    if (n_rows > 0) pf_cp16(dst, a.qrot + row_index(min(r, n_rows - 1)) * 2 + 8 * piece);
    else pt_sts128(dst, 0u, 0u, 0u, 0u);
  }
  asm volatile("cp.async.commit_group;" ::: "memory");
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();   // Q' is staged, tensor memory is allocated
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  const int half = (warp >> 2) & 1, row = tid & 127;                            // of a row owner: its side of the tokens and of the output
  const uint32_t trow = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);        // its tensor-memory lane
  if (warp < kPcOwners) {   // the values by one half of the owners, the residuals by the other
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
      const uint4* src = reinterpret_cast<const uint4*>(smem + kPtKv + row * (2 * kPtQStride * 2) + half * (kPtQStride * 2) + c * 128);
      uint32_t v[32];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 w = src[i];
        v[4 * i] = w.x; v[4 * i + 1] = w.y; v[4 * i + 2] = w.z; v[4 * i + 3] = w.w;
      }
      tc_st32u(trow + (half ? kPtTmQlo : kPtTmQhi) + 32 * c, v);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  }
  __syncthreads();   // Q' is in tensor memory; the staging is dead: the stages may be written
  pt_cluster_sync();   // both CTAs' barriers are initialised and both halves of Q' are in place
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // where this CTA's warps announce themselves: the barriers of the even CTA
  const uint32_t to_leader = pt_mapa(sb + kPtBase, 0u) - (sb + kPtBase);   // + a local shared address: that place in the even CTA (cluster window)

  float l_run = 0.f, m_run = -CUDART_INF_F;   // row owners: this thread's share of the row's denominator, and the row's reference
  float* row_max = reinterpret_cast<float*>(smem + kPcMax);   // [block parity][half][row]
  if (warp < kPcOwners) {
    // ================= row owners: softmax of row `row`, tokens 32 half .. + 31 of every block =================
    bool fail = false;   // of this warp; the owners leave together, at the barrier of a block
    for (int jb = 0; jb < n_blocks; ++jb) {
      const int t = jb % kPtScores;
      if (!fail) fail = !__all_sync(0xffffffffu, tc_mbar_wait(sb + kPtBarS + 8 * t, (uint32_t)(jb / kPtScores) & 1u, abort_flag));
      float s[32], mx = -CUDART_INF_F;
      if (!fail) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tc_ld32(trow + kPtTmS + 64 * t + 32 * half, s);
        const int t0 = (jb0 + jb) * kTokenBlock + 32 * half;
        if (t0 + 32 > len) {
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i] = t0 + i < len ? s[i] : -CUDART_INF_F;
        }
        float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};   // four chains: no 32-long dependency
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
#pragma unroll
          for (int c = 0; c < 4; ++c) mx4[c] = fmaxf(mx4[c], fmaxf(s[i + 2 * c], s[i + 2 * c + 1]));
        }
        mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        row_max[((jb & 1) * 2 + half) * 128 + row] = mx;
      }
      // both halves' maxima are there, and both have read the scores whose columns P takes
      if (pc_owners_failed(fail)) break;
      mx = fmaxf(mx, row_max[((jb & 1) * 2 + (half ^ 1)) * 128 + row]);
      const bool grow = mx > m_run + kPxMost || (m_run == -CUDART_INF_F && mx > -CUDART_INF_F);   // lazy reference: see kPxBelow
      if (__any_sync(0xffffffffu, grow)) {
        const float m_new = grow ? mx - kPxBelow : m_run;
        const float corr = m_run == -CUDART_INF_F ? 1.f : fast_exp2(m_run - m_new);   // nothing accumulated yet: nothing to scale
        if (jb > 0) {
          // the value MMAs up to block jb - 1 must have completed before the accumulator is touched
          fail = !__all_sync(0xffffffffu, tc_mbar_wait(sb + kPtBarPv + 8 * ((jb - 1) % kPtStages), (uint32_t)((jb - 1) / kPtStages) & 1u, abort_flag));
          if (fail) continue;   // to the next block's barrier
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
          for (int c = 0; c < 2; ++c) {
            float o[32];
            tc_ld32(trow + kPtTmO + 64 * half + 32 * c, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= corr;
            tc_st32(trow + kPtTmO + 64 * half + 32 * c, o);
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
        l_run *= corr;
        m_run = m_new;
      }
      const float m_use = m_run == -CUDART_INF_F ? 0.f : m_run;   // only scores of -inf so far: every p is 0
      // P_jb takes the first 32 columns of the accumulator it was computed from, this half 16 of them: the value MMA of block
      // jb - kPtScores, which read them last, was issued before the score MMAs that were waited for
      float sum4[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t pw[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float x0, x1;
        pt_add2(s[2 * e], s[2 * e + 1], -m_use, -m_use, x0, x1);
        x0 = fast_exp2(x0);
        x1 = fast_exp2(x1);
        pw[e] = as_u32(__floats2half2_rn(x0, x1));
        // the denominator, before the rounding to fp16: see kPxBelow
        pt_add2(sum4[2 * (e & 1)], sum4[2 * (e & 1) + 1], x0, x1, sum4[2 * (e & 1)], sum4[2 * (e & 1) + 1]);
      }
      tc_st16u_nowait(trow + kPtTmS + 64 * t + 16 * half, pw);
      l_run += (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) pt_arrive_cluster(sb + kPtBarP + 8 * t + to_leader);
    }
  } else if (warp < kPcFetchWarp) {
    // ================= decoders: packed block -> K_hat hi / lo, V_hat^T =================
    // Pieces of 1 / kPcGroups of this CTA's half of a block, counted through all blocks, go to the decoder warps in turn.  A piece is twice
    // 16 coordinates of 32 lanes = 8 tokens x 4 16-blocks: pieces 0-3 both halves of the coordinates of the keys of tokens 32 rank ..
    // + 31, pieces 4-7 the values of coordinates 64 rank .. + 63 of all 64 tokens.
    // (256 rows over 65536 tokens: 523 us with windows behind, 555 with pieces of half the size.)
    const int dw = warp - kPcOwners, bi = lane >> 3, t8 = lane & 7;
    const uint32_t rep = (uint32_t)(lane & 15) * 8u, t1 = (sb + kPtT1) | rep, ub = (sb + kPtU) | rep;
    const uint32_t swz = (uint32_t)(t8 * 128 + (((2 * bi) ^ t8) << 4));   // chunk 2 bi of a row's 64-coordinate half, swizzled by the row
    int ready = -1;   // the last block known to have landed and to have a stage
    for (int n = dw; n < kPcGroups * n_blocks; n += kPcDecoders) {
      const int jb = n / kPcGroups, i = n % kPcGroups, st = jb % kPtStages, buf = jb % kPtRawBufs;
      bool ok = true;
      if (jb != ready) {
        // stage st is free once the value MMA of block jb - kPtStages has completed (it also covers that block's score MMAs)
        if (jb >= kPtStages) ok = tc_mbar_wait(sb + kPtBarPv + 8 * st, (uint32_t)(jb / kPtStages - 1) & 1u, abort_flag);
        if (ok) ok = tc_mbar_wait(sb + kPtBarRawFull + 8 * buf, (uint32_t)(jb / kPtRawBufs) & 1u, abort_flag);
        ready = jb;
      }
      if (!__all_sync(0xffffffffu, ok)) break;
      const bool is_v = i >= kPcGroups / 2;
      const uint32_t raw = sb + kPtRaw + buf * kPtRawBytes + (is_v ? kBlockBytes128 : 0);
      if (!is_v) {
        const int tok = 8 * ((i & 3) + 4 * (int)crank) + t8;
        const bool live = (jb0 + jb) * kTokenBlock + tok < len;   // stale bytes past the sequence end must not reach the MMAs
        const uint32_t c4w = lds16(raw + kO4 + tok * 2) >> (2 * bi);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          const int blk = 4 * side + bi;
          const uint32_t l1 = lds32(raw + tok * 32 + blk * 4);
          const uint32_t c2 = lds8(raw + kO2 + tok * 8 + blk);
          const uint32_t c3 = lds8(raw + kO3 + tok * 4 + (blk >> 1)) >> (4 * (bi & 1));
          const uint32_t rbits = lds16(raw + kORad + tok * 16 + blk * 2);
          const uint32_t rr = live ? rbits | (rbits << 16) : 0u;
          const BlockRef ref = make_block_ref(l1, c2, c3, (c4w >> (8 * side)) & 3u, as_h2(rr), ub);
          // the key as an unevaluated sum hi + lo, coordinates in the order of the lookups: (4s, 4s+2), (4s+1, 4s+3)
          __half2 h[8], l[8];
          sub_block_hilo<0>(ref, t1, h[0], h[1], l[0], l[1]);
          sub_block_hilo<1>(ref, t1, h[2], h[3], l[2], l[3]);
          sub_block_hilo<2>(ref, t1, h[4], h[5], l[4], l[5]);
          sub_block_hilo<3>(ref, t1, h[6], h[7], l[6], l[7]);
          const uint32_t dst = sb + kPtKv + st * kPtStage + side * kPtKHalf + (i & 3) * 1024 + swz;
          pt_sts128(dst, as_u32(h[0]), as_u32(h[1]), as_u32(h[2]), as_u32(h[3]));
          pt_sts128(dst ^ 16u, as_u32(h[4]), as_u32(h[5]), as_u32(h[6]), as_u32(h[7]));
          pt_sts128(dst + kPtKLo, as_u32(l[0]), as_u32(l[1]), as_u32(l[2]), as_u32(l[3]));
          pt_sts128((dst + kPtKLo) ^ 16u, as_u32(l[4]), as_u32(l[5]), as_u32(l[6]), as_u32(l[7]));
        }
      } else {
        const int blk = 4 * (int)crank + bi;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tok = 8 * ((i & 3) + 4 * e) + t8;
          const bool live = (jb0 + jb) * kTokenBlock + tok < len;
          const uint32_t l1 = lds32(raw + tok * 32 + blk * 4);
          const uint32_t c2 = lds8(raw + kO2 + tok * 8 + blk);
          const uint32_t c3 = lds8(raw + kO3 + tok * 4 + (blk >> 1)) >> (4 * (bi & 1));
          const uint32_t c4 = (lds16(raw + kO4 + tok * 2) >> (2 * blk)) & 3u;
          const uint32_t rbits = lds16(raw + kORad + tok * 16 + blk * 2);
          const uint32_t rr = live ? rbits | (rbits << 16) : 0u;
          const BlockRef ref = make_block_ref(l1, c2, c3, c4, as_h2(rr), ub);
          __half2 x[4], y[4];
          sub_block_h2<0>(ref, t1, x[0], y[0]);
          sub_block_h2<1>(ref, t1, x[1], y[1]);
          sub_block_h2<2>(ref, t1, x[2], y[2]);
          sub_block_h2<3>(ref, t1, x[3], y[3]);
          // coordinates in natural order: (4s, 4s+1) = (x.lo, y.lo), (4s+2, 4s+3) = (x.hi, y.hi)
          uint32_t w[8];
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            w[2 * s] = __byte_perm(as_u32(x[s]), as_u32(y[s]), 0x5410);
            w[2 * s + 1] = __byte_perm(as_u32(x[s]), as_u32(y[s]), 0x7632);
          }
          const uint32_t dst = sb + kPtKv + st * kPtStage + kPtKTile + ((i & 3) + 4 * e) * 1024 + swz;
          pt_sts128(dst, w[0], w[1], w[2], w[3]);
          pt_sts128(dst ^ 16u, w[4], w[5], w[6], w[7]);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        pt_arrive_cluster(sb + kPtBarKv + 8 * st + to_leader);
        tc_mbar_arrive(sb + kPtBarRawEmpty + 8 * buf);
      }
    }
  } else if (warp == kPcFetchWarp) {
    // ================= packed blocks on their way: as many as there are buffers, each requested as soon as one is free =================
    if (lane == 0) {
      int fetched = min(kPtRawBufs, n_blocks);
      for (; fetched < n_blocks; ++fetched) {
        if (!tc_mbar_wait(sb + kPtBarRawEmpty + 8 * (fetched % kPtRawBufs), (uint32_t)(fetched / kPtRawBufs - 1) & 1u, abort_flag)) break;
        request(fetched);
      }
      for (int f = max(0, fetched - kPtRawBufs); f < fetched; ++f)   // no copy may be in flight when the CTA ends
        for (int i = 0; i < (1 << 20) && !tc_mbar_try(sb + kPtBarRawFull + 8 * (f % kPtRawBufs), (uint32_t)(f / kPtRawBufs) & 1u); ++i)
          __nanosleep(32);
    }
  } else if (leader) {
    // ================= MMA issuer =================
    // The whole warp goes through the loop and one elected lane issues: the operands of the MMAs are then warp-uniform values.
    // From a single thread's registers every MMA took 60 cycles to issue, more than it runs.
    // the value operand is MN-major: [token][coordinate] rows of 64 coordinates, one half per CTA
    constexpr uint32_t idesc_qk = tc_idesc(false, 256, 64);   // 64 tokens
    constexpr uint32_t idesc_pv = tc_idesc(false, 256, 128) | (1u << 16);
    uint64_t vdesc_hi = (uint64_t)(1024 >> 4) << 32;   // stride between groups of 8 tokens
    vdesc_hi |= (uint64_t)1 << 46;
    vdesc_hi |= (uint64_t)2 << 61;
    const uint32_t vdesc_lbo = (8192u >> 4) << 16;     // leading-dimension offset: the next 64 coordinates
    const uint64_t desc_hi = tc_smem_desc(0u) & 0xFFFFFFFF00000000ull;
    const int blocks = __shfl_sync(0xffffffffu, n_blocks, 0);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
    auto issue_pv = [&](int jb) {   // O (+)= P_jb V_hat_jb
      const int t = jb % kPtScores, st = jb % kPtStages;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t v_lo = ((kPtKv + st * kPtStage + kPtKTile) >> 4) | vdesc_lbo;
      if (tc_elect()) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)   // 16 tokens = 8 columns of P = 16 rows of 128 bytes of V_hat per step
          tc_mma_ts_pair(tm + kPtTmO, tm + kPtTmS + 64 * t + 8 * kk, vdesc_hi | (v_lo + 128 * kk), idesc_pv, (jb > 0 || kk > 0) ? 1u : 0u);
        tc_commit_pair(sb + kPtBarPv + 8 * st);   // the stage is free, the output accumulator holds block jb
      }
    };
    auto issue_qk = [&](int jb) {   // S_jb = Q'lo K_hi^T + Q'hi K_lo^T + Q'hi K_hi^T, the small terms first
      const int t = jb % kPtScores, st = jb % kPtStages;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t kb = (uint32_t)tc_smem_desc(kPtKv + st * kPtStage);
      if (tc_elect()) {
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          const uint32_t qa = tm + (term == 0 ? kPtTmQlo : kPtTmQhi);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {   // 16 k values = 8 columns of Q' per step; step ks: half ks >> 2, 32 bytes per step
            const uint32_t koff = (uint32_t)((ks >> 2) * kPtKHalf + (ks & 3) * 32 + (term == 1 ? kPtKLo : 0)) >> 4;
            tc_mma_ts_pair(tm + kPtTmS + 64 * t, qa + 8 * ks, desc_hi | (kb + koff), idesc_qk, (term | ks) ? 1u : 0u);
          }
        }
        tc_commit_pair(sb + kPtBarS + 8 * t);
      }
    };
    // A fixed order, so that the warp sleeps in its waits and leaves its scheduler to the others (looking at both barriers in turn cost a
    // fifth of it): the score MMAs run kPtScores - 1 blocks ahead of the value MMAs.  Accumulator t is free for block jb once the value
    // MMA of block jb - kPtScores, which reads P from its columns, has been issued (MMAs of one thread execute in order).
    bool ok = true;
    for (int jb = 1 - kPtScores; jb < blocks && ok; ++jb) {
      if (jb >= 0) {
        ok = __all_sync(0xffffffffu, tc_mbar_wait(sb + kPtBarP + 8 * (jb % kPtScores), (uint32_t)(jb / kPtScores) & 1u, abort_flag));
        if (ok) issue_pv(jb);
      }
      const int qk = jb + kPtScores - 1;
      if (ok && qk < blocks) {
        ok = __all_sync(0xffffffffu, tc_mbar_wait(sb + kPtBarKv + 8 * (qk % kPtStages), (uint32_t)(qk / kPtStages) & 1u, abort_flag));
        if (ok) issue_qk(qk);
      }
    }
    if (blocks > 0) {
      // every MMA issued above has completed when this commit arrives (nothing was issued without blocks: no commit)
      if (tc_elect()) tc_commit_pair(sb + kPtBarDrain);
      bool drained = false;
      for (int i = 0; i < (1 << 20) && !drained; ++i) {
        drained = tc_mbar_try(sb + kPtBarDrain, 0);
        if (!drained) __nanosleep(32);
      }
      if (!drained) *abort_flag = 1;
    }
    __syncwarp();
    if (lane == 0 && *abort_flag)   // tell the other CTA, whose warps wait for commits that will not come
      asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(kPtMisc + 4 - kPtBase + pt_mapa(sb + kPtBase, 1u)), "r"(1u) : "memory");
  } else if (lane == 0) {
    // the odd CTA of a pair: its operands are read until the even CTA's last commit arrives here too
    if (n_blocks > 0) {
      bool drained = false;
      for (int i = 0; i < kTcSpin && !drained && !*abort_flag; ++i) {
        drained = tc_mbar_try(sb + kPtBarDrain, 0);
        if (!drained) __nanosleep(64);
      }
      if (!drained) *abort_flag = 1;
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();   // all MMAs have completed (the issuer waited for its last commit), the stages are idle
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const bool aborted = *abort_flag != 0;
  // ---- normalise; prefix_unrotate_kernel merges the ranges' parts and rotates back
  float* osm = reinterpret_cast<float*>(smem + kPtKv);
  if (warp < kPcOwners) row_max[half * 128 + row] = l_run;
  __syncthreads();
  if (warp < kPcOwners) {
    const float l = row_max[row] + row_max[128 + row];
    const float inv = (!aborted && l > 0.f) ? 1.f / l : 0.f;
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
      float o[32];
      if (n_blocks > 0 && !aborted) {
        tc_ld32(trow + kPtTmO + 64 * half + 32 * c, o);
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 32; i += 4)
        *reinterpret_cast<float4*>(osm + row * kPtOStride + 64 * half + 32 * c + i) = make_float4(o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
    }
    if (half == 0 && row < n_rows)   // scores are in the log2 domain
      a.part_lse[(int64_t)split * a.batch * a.n_q_heads + row_index(row) / 128] =
          l > 0.f ? (m_run + log2f(l)) * 0.693147180559945309f : l == 0.f ? -CUDART_INF_F : l;   // NaN stays NaN
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  }
  __syncthreads();
  // Neither CTA may release tensor memory or leave while the other may still arrive on its barriers or
  // have its operands read: both have drained here.
  pt_cluster_sync();
  if (warp == kPcMmaWarp) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
  }
  if (tid == 0 && aborted) set_status(a.status, PQ_ERR_TIMEOUT);
  for (int i = tid; i < n_rows * 32; i += kPcThreads)
    *reinterpret_cast<float4*>(a.part_out + (int64_t)split * a.batch * a.n_q_heads * 128 + row_index(i >> 5) + 4 * (i & 31)) =
        *reinterpret_cast<const float4*>(osm + (i >> 5) * kPtOStride + 4 * (i & 31));
}

}  // namespace pq
