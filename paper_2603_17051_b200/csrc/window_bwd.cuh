// Backward of attention with a sliding window and sinks (window_common.cuh), nothing detached.
//   dQ     a query tile stationary, over the key tiles that it sees:    dQ = scale * sum dS K
//   dK/dV  a key tile stationary, over the query tiles of all the heads that share it and see it:
//          dV = sum P^T dO, dK = scale * sum dS^T Q
// with P = exp(S - LSE), dS = P o (dP - delta), as in the dense kernels (attn_bwd.cuh), whose tensor-memory layouts, operand
// forms and hand-offs these two have: see there.  Both in one launch, a CTA per tile, the long jobs first: the key tiles of the
// sinks, which every query sees (several CTAs to a tile where it would take longer than everything else), the other key tiles,
// the query tiles.  Tiles of which a row sees only a part are masked bit by bit, P and dS by selection, so that what a masked
// place holds, NaN included, ends there; rows behind a sequence's end are cleared in shared memory where they are operands.
// Inside a sequence a NaN or infinity in K, Q or dO would still reach the rows of a masked tile that do not see it (0 * NaN):
// a tile whose gradients are not finite is done again by the formula, on the ordinary cores (slow and rare).
// Every accumulator belongs to one CTA: results do not depend on the order of anything.
// Bound: the hand-offs S -> P -> dP -> dS of one tile at a time and the tensor pipe (72 %): 32760 tokens of a video (window_fwd.cuh) in
// 8450 us: 995 TFLOP/s of five products a pair, 1390 of the seven that two passes make; 16384 causal tokens, 12 heads: 2120 us at head_dim 128, 1630 at 64.  Clocks per tile at 128: dQ
// about 2190 (exponentials 1050, dS 500, waits 400), dK/dV 2750 (1170, 760, 500).  Skipping the exponentials of 32 by 32 pairs that
// are masked, as the forward does, gave 12.5 -> 11.5 us for 300 tokens and 1628 -> 1775 for 16384: the branch costs the full tiles' schedule.
// Precision: bf16 products, fp32 sums; P and dS are rounded to bf16 (half a step, 2^-8 of each term at most) as operands of the
// second products.
#pragma once
#include "attn_bwd.cuh"
#include "sparse_common.cuh"
#include "window_fwd.cuh"

namespace astro {

struct WinBwdArgs {
  const __nv_bfloat16 *q, *k, *v, *d_o;
  WinStrides qs, ks, vs;
  const float *lse, *delta;       // [B, H, n]
  __nv_bfloat16 *dq, *dk, *dv;    // [B, n, H or KVH, D]
  WinMask mask;
  int heads, kv_heads, group, lists, kv_lists, tiles;   // lists = batch * heads, kv_lists = batch * kv_heads
  Divisor by_heads, by_kv_heads, by_group;
  WinOrder q_order, k_order;      // of the query tiles and of the key tiles behind the front ones
  int front;                      // key tiles of the sinks, where they come first
  int shares;                     // CTAs that share each of them
  float* parts;                   // [front][list][share][dK | dV][128][D] when shares > 1
  float scale;
};
constexpr int kWinGroups = 2;                             // softmax groups of 128 threads, 32 columns of a tile each
constexpr int kWinBwdThreads = 128 * kWinGroups + 64;     // + MMA, loads

// 32 accumulator columns of the lane's row times `mult`, zeros where the row is not live, as bf16; whether all are finite.
__device__ __forceinline__ bool win_store_row32(uint32_t taddr, float mult, bool live, const QuadRows& rows, int col0, int lane) {
  uint32_t r[32];
  tmem_ld32(taddr, r);
  tmem_wait_ld();
  uint64_t chk2 = f32x2(0.f, 0.f);
  win_store_slice(r, mult, live, chk2, rows, col0, lane);
  return !live || fwd_all_finite(chk2);
}

// delta of rows that see few keys from the weights, sum_j p_ij dO_i . v_j, instead of dO_i . O_i with the rounded O: where one of a few
// keys has nearly all the weight, dS is far smaller than delta, and half a step of O's (2^-8 of delta) is then per cents of it.
// Where rows see many keys, those with large gradients outweigh such a one; where all of them see few, because the window is narrow or the
// sequence short, it can be all of the result.  So: every row where window and sinks are kWinFewKeys keys or fewer, and the samples
// of that length or less of a batch whose rows see more.
// A warp per 8 queries of one head of one sample, S^T = K Q^T and dP^T = V dO^T for 16 keys a step by mma.sync (the elements of a head
// are summed in the order in which lanes load them).  L2: 16384 tokens, 12 heads of 128, a window of 64 in 100 us (of a
// window of 8 in 48) beside 215 for the gradients, where dO . O takes 21; for 2 x 64 tokens of 12 heads the backward takes 14.3 us, 33.3
// with a warp per query.
constexpr int kWinFewKeys = 64;
template <int D>
__global__ void __launch_bounds__(128) win_few_delta_kernel(const WinBwdArgs a, const int rows, const int longest, float* delta) {
  constexpr int kPieces = D / 64;
  dependents_may_start();
  const long long groups = (rows + 7) / 8, at = blockIdx.x * 4ll + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long list = at / groups;
  const int i0 = static_cast<int>(at - list * groups) * 8;
  const int b = static_cast<int>(list / a.heads), h = static_cast<int>(list - static_cast<long long>(b) * a.heads);
  const int len = list < a.lists ? a.mask.length(b) : 0;
  if (len > longest || i0 >= len) {
    dependency_wait();   // what follows this launch waits for this one alone
    return;
  }
  // a lane's pieces of a row: elements 8 (t + 4 (2 c + x)) .. at [c][x], 64 contiguous bytes per row and load
  auto load_row = [&](const __nv_bfloat16* row, uint4 (&w)[kPieces][2]) {
#pragma unroll
    for (int c = 0; c < kPieces; ++c)
#pragma unroll
      for (int x = 0; x < 2; ++x) w[c][x] = reinterpret_cast<const uint4*>(row)[t + 4 * (2 * c + x)];
  };
  uint4 q[kPieces][2], d_o[kPieces][2];
  const int own = min(i0 + g, len - 1);   // the query of the operands
  load_row(a.q + b * a.qs.b + own * a.qs.t + h * a.qs.h, q);
  load_row(a.d_o + ((static_cast<size_t>(b) * a.mask.n + own) * a.heads + h) * D, d_o);
  // the queries of the results: 2t, 2t + 1
  int lo[2], hi[2], from, unused, end;
  float lse2[2], sum[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int i = min(i0 + 2 * t + c, len - 1);
    a.mask.keys_of(i, len, lo[c], hi[c]);
    lse2[c] = a.lse[(static_cast<size_t>(b) * a.heads + h) * a.mask.n + i] * kLog2e;
  }
  a.mask.keys_of(i0, len, from, unused);
  a.mask.keys_of(min(i0 + 7, len - 1), len, unused, end);
  const int sink = min(a.mask.sink, from), keys = sink + end - from;   // [0, sink) and [from, end)
  const float scale_log2 = a.scale * kLog2e;
  const __nv_bfloat16 *kb = a.k + b * a.ks.b + (h / a.group) * a.ks.h, *vb = a.v + b * a.vs.b + (h / a.group) * a.vs.h;
  auto key = [&](int x) { return x < sink ? x : from + x - sink; };
  for (int x0 = 0; x0 < keys; x0 += 16) {
    float s[4] = {0.f, 0.f, 0.f, 0.f}, dp[4] = {0.f, 0.f, 0.f, 0.f};
    const long long j0 = key(min(x0 + g, keys - 1)), j1 = key(min(x0 + g + 8, keys - 1));
    uint4 k0[kPieces][2], k1[kPieces][2], v0[kPieces][2], v1[kPieces][2];
    auto products = [&](const uint4 (&x)[kPieces][2], const uint4 (&y)[kPieces][2], const uint4 (&with)[kPieces][2], float (&to)[4]) {
#pragma unroll
      for (int c = 0; c < kPieces; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma_16x8x16<true>(to, x[c][i].x, y[c][i].x, x[c][i].y, y[c][i].y, with[c][i].x, with[c][i].y);
          mma_16x8x16<true>(to, x[c][i].z, y[c][i].z, x[c][i].w, y[c][i].w, with[c][i].z, with[c][i].w);
        }
    };
    load_row(kb + j0 * a.ks.t, k0);
    load_row(kb + j1 * a.ks.t, k1);
    load_row(vb + j0 * a.vs.t, v0);
    load_row(vb + j1 * a.vs.t, v1);
    products(k0, k1, q, s);
    products(v0, v1, d_o, dp);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at_key = x0 + g + 8 * (e / 2), j = key(at_key), c = e % 2;
      const bool sees = at_key < keys && j < hi[c] && (j < a.mask.sink || j >= lo[c]);
      sum[c] += sees ? fast_exp2(s[e] * scale_log2 - lse2[c]) * dp[e] : 0.f;
    }
  }
  dependency_wait();   // this launch may follow one that writes delta of every row
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int d = 4; d < 32; d *= 2) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], d);
    const int i = i0 + 2 * t + c;
    if (g == 0 && i < len) delta[(static_cast<size_t>(b) * a.heads + h) * a.mask.n + i] = sum[c];
  }
}

// ------------------------------------------------------------------------------------------ dQ
// One row of dQ by the formula: eight lanes per key, four keys at a time.
template <int D>
__device__ __noinline__ void win_careful_dq(const WinBwdArgs& a, int qt, int h, int b, int warp, int lane) {
  constexpr int kPer = D / 8;
  const int len = a.mask.length(b), part = lane & 7, slot = lane >> 3;
  for (int r = warp; r < kTile; r += kWinBwdThreads / 32) {
    const int row = qt * kTile + r;
    if (row >= len) break;
    const size_t stat = (static_cast<size_t>(b) * a.heads + h) * a.mask.n + row;
    const float lse2 = a.lse[stat] * kLog2e, delta = a.delta[stat], scale_log2 = a.scale * kLog2e;
    const bool alone = a.mask.one_key(row, len);
    const __nv_bfloat16* qp = a.q + b * a.qs.b + row * a.qs.t + h * a.qs.h + part * kPer;
    const size_t at = ((static_cast<size_t>(b) * a.mask.n + row) * a.heads + h) * D + part * kPer;
    float acc[kPer], q[kPer], g[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      acc[e] = 0.f;
      q[e] = __bfloat162float(qp[e]);
      g[e] = __bfloat162float(a.d_o[at + e]);
    }
    bool lost = false;
    int lo, hi;
    a.mask.keys_of(row, len, lo, hi);
    const int sink = min(min(a.mask.sink, hi), lo), keys = sink + hi - lo;
    const __nv_bfloat16* kb = a.k + b * a.ks.b + (h / a.group) * a.ks.h + part * kPer;
    const __nv_bfloat16* vb = a.v + b * a.vs.b + (h / a.group) * a.vs.h + part * kPer;
    for (int x = 0; x < keys; x += 4) {
      const bool there = x + slot < keys;
      const int y = there ? x + slot : keys - 1, j = y < sink ? y : lo + y - sink;
      float s = 0.f, dp = 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        s = fmaf(q[e], __bfloat162float(kb[j * a.ks.t + e]), s);
        dp = fmaf(g[e], __bfloat162float(vb[j * a.vs.t + e]), dp);
      }
#pragma unroll
      for (int d = 1; d < 8; d *= 2) {
        s += __shfl_xor_sync(0xffffffffu, s, d);
        dp += __shfl_xor_sync(0xffffffffu, dp, d);
      }
      if ((x & 127) == 0 && __any_sync(0xffffffffu, lost)) break;   // NaN in every element: nothing to add to that
      if (there) {
        float ds = fast_exp2(s * scale_log2 - lse2) * (dp - delta);
        if (alone && fabsf(ds) < INFINITY) ds = 0.f;
        lost = lost || isnan(ds);
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = fmaf(ds, __bfloat162float(kb[j * a.ks.t + e]), acc[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
#pragma unroll
      for (int d = 8; d < 32; d *= 2) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], d);
      if (slot == 0) a.dq[at + e] = __float2bfloat16_rn(acc[e] * a.scale);
    }
  }
}

template <int D>
__device__ __forceinline__ void win_bwd_dq(uint8_t* smem_raw, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CUtensorMap& tm_do,
                                           const WinBwdArgs& a, const int qt, const int list) {
  uint8_t* smem = align_1024(smem_raw);
  uint8_t* sdO = smem + DqSmem<D>::kdO;
  uint8_t* sK = smem + DqSmem<D>::kK;
  uint8_t* sV = smem + DqSmem<D>::kV;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + DqSmem<D>::kBars);
  uint64_t *kv0_full = bars, *qt_full = bars + 1, *rs = bars + 2, *rb = bars + 6, *s_full = bars + 10, *b_done = bars + 11,
           *dq_full = bars + 13, *landed = bars + 14;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 15);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = a.by_heads.quot(list), h = list - b * a.heads;
  const int q0 = qt * kTile, len = a.mask.length(b), kvh = a.by_group.quot(h);
  constexpr uint32_t kTmemCols = 512;
  constexpr uint32_t kColS = 0, kColdP = 128, kColdS = 256, kColQ = 320, kColdQ = 384;
  constexpr int kMmaWarp = 4 * kWinGroups, kTmaWarp = kMmaWarp + 1, kCols = kTile / kWinGroups, NL = kCols / 32;

  if (q0 >= len) {   // nothing but zeros, the same for the whole CTA
    dependency_wait();
    if (warp < 8) {
      const QuadRows rows = quad_rows(a.dq, b, h, a.mask.n, a.heads, D, q0 + (tid & 127));
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        uint4 zero[4] = {};
        store_quad_rows(zero, rows, (warp >> 2) * (D / 2) + c * 32, lane);
      }
    }
    return;
  }
  WinTiles tiles;
  tiles.set(a.mask, q0, len);
  const int n_tiles = tiles.count();

  if (warp == kTmaWarp && lane == 0) { tma_prefetch_desc(&tm_k); tma_prefetch_desc(&tm_v); tma_prefetch_desc(&tm_do); }
  if (tid < 15) {
    // qt_full: one arrival per warp and 64 elements; rs, rb: bytes and warps
    mbar_init(bars + tid, tid == 1 ? 4 * (D / 64) : tid >= 2 && tid < 10 ? 1 + 4 * kWinGroups : 1);
    fence_mbar_init();
  }
  if (tid == 0) *abort_flag = 0;
  fence_proxy_async_smem();
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_holder;
  bool redo = false;

  if (warp == kTmaWarp) {
    int kt = tiles.first();
    // K of a tile that straddles the sequence's end: its rows behind it are cleared before anyone is told (dS is 0 there, but
    // 0 * NaN would reach dQ).  It is the last tile, so at most once.
    auto load_kv = [&](int t, uint64_t* k_bar, uint64_t* v_bar, bool k_counted) {
      uint8_t *k_dst = sK + (t % kDqKStages) * TileGeom<D>::kBytes, *v_dst = sV + (t % kDqVStages) * TileGeom<D>::kBytes;
      const bool straddles = kt * kTile + kTile > len && len < a.mask.n;
      bool ok = true;
      if (lane == 0) tma_load_tile<D>(v_dst, &tm_v, v_bar, kt * kTile, kvh, b);
      if (straddles) {
        if (lane == 0) {
          mbar_arrive_expect_tx(landed, TileGeom<D>::kBytes);
          tma_load_tile<D>(k_dst, &tm_k, landed, kt * kTile, kvh, b);
        }
        ok = mbar_wait_ok(landed, 0, abort_flag);
        zero_rows_by_warp<D>(k_dst, len - kt * kTile, lane);
        if (lane == 0 && k_counted) mbar_arrive(k_bar);
      } else if (lane == 0) {
        if (k_counted) mbar_arrive_expect_tx(k_bar, TileGeom<D>::kBytes);
        tma_load_tile<D>(k_dst, &tm_k, k_bar, kt * kTile, kvh, b);
      }
      kt = tiles.next(kt);
      return ok;
    };
    const bool k0_straddles = kt * kTile + kTile > len && len < a.mask.n;
    // kv0_full counts one arrival: it comes with the bytes, or behind the clearing where there is any
    if (lane == 0) {
      if (!k0_straddles) mbar_arrive_expect_tx(kv0_full, 3 * TileGeom<D>::kBytes);
      else asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(kv0_full)), "r"(2 * TileGeom<D>::kBytes) : "memory");
      tma_load_tile<D>(sdO, &tm_do, kv0_full, q0, h, b);
    }
    __syncwarp();
    bool ok = load_kv(0, kv0_full, kv0_full, false);
    if (k0_straddles && lane == 0) mbar_arrive(kv0_full);
    for (int t = 1; ok && t <= n_tiles; ++t) {
      // commit t-1 of b_done: dQ(t-3) and dP(t-2) are done, the K stage and the V stage of tile t are free
      if (t >= 2 && !mbar_wait_ok(b_done + ((t - 1) & 1), ((t - 2) >> 1) & 1, abort_flag)) break;
      if (t < n_tiles) {
        if (lane == 0) mbar_arrive_expect_tx(rb + (t - 1) % 4, TileGeom<D>::kBytes);
        __syncwarp();
        ok = load_kv(t, rs + (t - 1) % 4, rb + (t - 1) % 4, true);
      } else if (lane == 0) {
        mbar_arrive(rb + (t - 1) % 4);   // the last tile's burst waits for no bytes (its rs is never awaited)
      }
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      constexpr uint32_t idesc_s = make_idesc_bf16(kTile, kTile, false, false);
      const uint64_t k_desc0 = desc_kmajor(smem_u32(sK));
      auto issue_s = [&](int j) {
        const uint64_t k_desc = desc_step(k_desc0, (j % kDqKStages) * TileGeom<D>::kBytes);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_ts(tmem_base + kColS, tmem_base + kColQ + k * 8,
                 desc_step(k_desc, (k >> 2) * TileGeom<D>::kBlockBytes + (k & 3) * 32), idesc_s, k > 0);
        mma_commit(s_full);
      };
      auto issue_dp = [&](int j) {
        mma_abT<D>(tmem_base + kColdP, smem_u32(sdO), smem_u32(sV + (j % kDqVStages) * TileGeom<D>::kBytes));
      };
      bool ok = mbar_wait_spin(qt_full, 0, abort_flag);
      ok = mbar_wait_spin(kv0_full, 0, abort_flag) && ok;
      tc_fence_after_sync();
      if (ok) {
        issue_s(0);
        issue_dp(0);
        mma_commit(b_done + 1);                       // commit 1
      }
      for (int j = 0; ok && j < n_tiles; ++j) {
        const bool more = j + 1 < n_tiles;
        if (more) {
          if (!mbar_wait_spin(rs + j % 4, (j / 4) & 1, abort_flag)) break;
          tc_fence_after_sync();
          issue_s(j + 1);
        }
        if (!mbar_wait_spin(rb + j % 4, (j / 4) & 1, abort_flag)) break;
        tc_fence_after_sync();
        if (more) issue_dp(j + 1);
        mma_pb<D, kTile>(tmem_base + kColdQ, tmem_base + kColdS, smem_u32(sK + (j % kDqKStages) * TileGeom<D>::kBytes), j > 0);
        mma_commit(b_done + (j & 1));                 // commit j + 2
      }
      mma_commit(dq_full);
    }
  } else {
    const int g = warp >> 2;
    const int r = tid & 127;
    const uint32_t tmem_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const int row = q0 + r;
    const bool live = row < len;
    const size_t stat_idx = (static_cast<size_t>(b) * a.heads + h) * a.mask.n + (live ? row : 0);
    {   // Q row -> tensor memory: group g writes elements [64g, 64g+64) of its row as 32 packed columns
      if (g * 64 < D) {
        uint32_t qr[32];
        const QuadRows q_rows = quad_rows_strided(a.q, a.qs, b, h, a.mask.n, row);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint4 ch[4];
          load_quad_rows(ch, q_rows, g * 64 + half * 32, lane);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            qr[16 * half + 4 * v] = ch[v].x; qr[16 * half + 4 * v + 1] = ch[v].y;
            qr[16 * half + 4 * v + 2] = ch[v].z; qr[16 * half + 4 * v + 3] = ch[v].w;
          }
        }
        tmem_st32(tmem_lane + kColQ + g * 32, qr);
        tmem_wait_st();
        tc_fence_before_sync();
        warp_arrive(qt_full, lane);
      }
    }
    dependency_wait();   // delta
    const float lse2 = live ? a.lse[stat_idx] * kLog2e : 0.f;
    const float delta_r = live ? a.delta[stat_idx] : 0.f;
    const float scale_log2 = a.scale * kLog2e;
    const uint64_t sc2 = f32x2(scale_log2, scale_log2), nl2 = f32x2(-lse2, -lse2), nd2 = f32x2(-delta_r, -delta_r);
    int lo = 0, hi = 0;
    // A row of one key has dS = 0, of which dP - delta would leave fp32's rounding: it sees nothing, unless it is NaN or infinite.
    const bool zero = a.mask.one_key(row, len) && fabsf(lse2) < INFINITY && fabsf(delta_r) < INFINITY;
    if (live && !zero) a.mask.keys_of(row, len, lo, hi);
    const int sink = min(a.mask.sink, hi);
    int kt = tiles.first();
    for (int j = 0; j < n_tiles; ++j, kt = tiles.next(kt)) {
      bool ok = mbar_wait_ok(s_full, j & 1, abort_flag);
      tc_fence_after_sync();
      uint32_t s[NL][32];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) tmem_ld32(tmem_lane + kColS + g * kCols + c2 * 32, s[c2]);
      tmem_wait_ld();
      tc_fence_before_sync();
      warp_arrive(rs + j % 4, lane);
      uint64_t p2[NL][16];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2)
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          float x0, x1;
          f32x2_split(fma2(f32x2(__uint_as_float(s[c2][c]), __uint_as_float(s[c2][c + 1])), sc2, nl2), x0, x1);
          p2[c2][c >> 1] = f32x2(fast_exp2(x0), fast_exp2(x1));
        }
      // commit j+1 of b_done: dP(j) is there, and dQ(j-1) has consumed the one dS buffer
      ok = mbar_wait_ok(b_done + ((j + 1) & 1), (j >> 1) & 1, abort_flag) && ok;
      tc_fence_after_sync();
      uint32_t dp[NL][32], ds[NL][16];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) tmem_ld32(tmem_lane + kColdP + g * kCols + c2 * 32, dp[c2]);
      tmem_wait_ld();
      if (tiles.full(kt)) {
#pragma unroll
        for (int c2 = 0; c2 < NL; ++c2)
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float d0, d1;
            f32x2_split(mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c2][c]), __uint_as_float(dp[c2][c + 1])), nd2)), d0, d1);
            ds[c2][c >> 1] = pack_bf16(d0, d1);
          }
      } else {
#pragma unroll
        for (int c2 = 0; c2 < NL; ++c2) {
          const int base = kt * kTile + g * kCols + c2 * 32;
          const uint32_t see = bits_below(sink, base) | (bits_below(hi, base) & ~bits_below(lo, base));
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float d0, d1;
            f32x2_split(mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c2][c]), __uint_as_float(dp[c2][c + 1])), nd2)), d0, d1);
            ds[c2][c >> 1] = pack_bf16((see >> c) & 1u ? d0 : 0.f, (see >> (c + 1)) & 1u ? d1 : 0.f);
          }
        }
      }
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) tmem_st16(tmem_lane + kColdS + g * (kCols / 2) + c2 * 16, ds[c2]);
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(rb + j % 4, lane);   // dS(j) stored; dP(j) was read before it, so its buffer is free as well
      if (!ok) break;
    }
    mbar_wait(dq_full, 0, abort_flag);
    tc_fence_after_sync();
    const QuadRows rows = quad_rows(a.dq, b, h, a.mask.n, a.heads, D, row);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      if (c % kWinGroups == g) redo = !win_store_row32(tmem_lane + kColdQ + c * 32, a.scale, live, rows, c * 32, lane) || redo;
  }

  settle_after_abort(abort_flag);
  tc_fence_before_sync();
  if (__syncthreads_or(redo) && !*abort_flag) win_careful_dq<D>(a, qt, h, b, warp, lane);
  if (warp == kMmaWarp) tmem_dealloc(tmem_base, kTmemCols);
}

// ------------------------------------------------------------------------------------------ dK, dV
// One row each of dK and dV by the formula: eight lanes per query, four queries at a time.
template <int D>
__device__ __noinline__ void win_careful_dkv(const WinBwdArgs& a, int kt, int kvh, int b, int warp, int lane, int first_row, int end_row) {
  constexpr int kPer = D / 8;
  const int len = a.mask.length(b), part = lane & 7, slot = lane >> 3;
  for (int r = first_row + warp; r < end_row; r += kWinBwdThreads / 32) {
    const int row = kt * kTile + r;
    if (row >= len) break;
    const float scale_log2 = a.scale * kLog2e;
    const __nv_bfloat16 *kp = a.k + b * a.ks.b + row * a.ks.t + kvh * a.ks.h + part * kPer,
                        *vp = a.v + b * a.vs.b + row * a.vs.t + kvh * a.vs.h + part * kPer;
    float dk[kPer], dv[kPer], k[kPer], v[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      dk[e] = dv[e] = 0.f;
      k[e] = __bfloat162float(kp[e]);
      v[e] = __bfloat162float(vp[e]);
    }
    int first, last;
    a.mask.queries_of(row, len, first, last);
    const bool alone = a.mask.one_key(row, len);
    for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h) {
      const size_t stat = (static_cast<size_t>(b) * a.heads + h) * a.mask.n;
      const __nv_bfloat16* qb = a.q + b * a.qs.b + h * a.qs.h + part * kPer;
      const __nv_bfloat16* gb = a.d_o + (static_cast<size_t>(b) * a.mask.n * a.heads + h) * D + part * kPer;
      const long long g_row = static_cast<long long>(a.heads) * D;
      for (int x = first; x < last; x += 4) {
        const bool there = x + slot < last;
        const int i = there ? x + slot : last - 1;
        float s = 0.f, dp = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          s = fmaf(k[e], __bfloat162float(qb[i * a.qs.t + e]), s);
          dp = fmaf(v[e], __bfloat162float(gb[i * g_row + e]), dp);
        }
#pragma unroll
        for (int d = 1; d < 8; d *= 2) {
          s += __shfl_xor_sync(0xffffffffu, s, d);
          dp += __shfl_xor_sync(0xffffffffu, dp, d);
        }
        if ((x - first & 127) == 0) {   // NaN in every element of both: nothing to add to that
          bool lost = true;
#pragma unroll
          for (int e = 0; e < kPer; ++e) lost = lost && isnan(dk[e]) && isnan(dv[e]);
          const uint32_t lanes = __ballot_sync(0xffffffffu, lost);   // all eight lanes of a slot
          if (((lanes & 0xffu) == 0xffu) || (lanes >> 8 & 0xffu) == 0xffu || (lanes >> 16 & 0xffu) == 0xffu || lanes >> 24 == 0xffu) break;
        }
        if (there) {
          const float p = fast_exp2(s * scale_log2 - a.lse[stat + i] * kLog2e);
          float ds = p * (dp - a.delta[stat + i]);
          if (alone && i == row && fabsf(ds) < INFINITY) ds = 0.f;
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            dk[e] = fmaf(ds, __bfloat162float(qb[i * a.qs.t + e]), dk[e]);
            dv[e] = fmaf(p, __bfloat162float(gb[i * g_row + e]), dv[e]);
          }
        }
      }
    }
    const size_t at = ((static_cast<size_t>(b) * a.mask.n + row) * a.kv_heads + kvh) * D + part * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
#pragma unroll
      for (int d = 8; d < 32; d *= 2) {
        dk[e] += __shfl_xor_sync(0xffffffffu, dk[e], d);
        dv[e] += __shfl_xor_sync(0xffffffffu, dv[e], d);
      }
      if (slot == 0) {
        a.dk[at + e] = __float2bfloat16_rn(dk[e] * a.scale);
        a.dv[at + e] = __float2bfloat16_rn(dv[e]);
      }
    }
  }
}

// acc[128 x D] (+)= A[128 x 128] B[128 x D], A as the softmax groups leave it: bf16 pairs, group g's from its own first column on.
template <int D>
__device__ __forceinline__ void win_mma_groups(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_smem, bool accumulate) {
  constexpr uint32_t idesc = make_idesc_bf16(kTile, D, false, true);
  constexpr int kCols = kTile / kWinGroups;
  const uint64_t b_desc = desc_mnmajor(b_smem, TileGeom<D>::kBlockBytes);
#pragma unroll
  for (int k = 0; k < kTile / 16; ++k)
    mma_ts(d_tmem, a_tmem + (k * 16 / kCols) * kCols + (k * 16 % kCols) / 2, desc_step(b_desc, k * 2048), idesc, (accumulate || k > 0) ? 1u : 0u);
}

// The dense kernel's hand-offs (a tile takes 2750 clocks: P^T 1170, dV and the next S^T 1024 behind it, the rest on the way), and at
// head_dim 64, where tensor memory has room, a second S^T buffer: S^T of the tile after the next is issued behind dV of this one, so
// the softmax warps never wait for it.
//   TMEM columns, head_dim 128:  S^T / P^T [0, 128)   dP^T / dS^T [128, 256)   dK [256, 384)   dV [384, 512)
//                 head_dim 64:   S^T / P^T [0, 256)   dP^T / dS^T [256, 384)   dK [384, 448)   dV [448, 512)
template <int D> struct WinDkvSmem {
  static constexpr int kSBufs = D == 128 ? 1 : 2;
  static constexpr int kStages = D == 128 ? 2 : 4;                        // of (Q, dO)
  static constexpr int kK = 0;
  static constexpr int kV = TileGeom<D>::kBytes;
  static constexpr int kQ = 2 * TileGeom<D>::kBytes;
  static constexpr int kdO = kQ + kStages * TileGeom<D>::kBytes;
  static constexpr int kStats = kdO + kStages * TileGeom<D>::kBytes;      // float [stages][2][128]: -lse*log2e, -delta
  static constexpr int kBars = kStats + kStages * 2 * kTile * 4;
  static constexpr int kTotal = kBars + 256 + 1024;
  static_assert((9 + 2 * kStages) * 8 + 8 <= 256, "barriers, tensor memory's address, abort flag");
};

template <int D>
__device__ __forceinline__ void win_bwd_dkv(uint8_t* smem_raw, const CUtensorMap& tm_q, const CUtensorMap& tm_do, const CUtensorMap& tm_k,
                                            const CUtensorMap& tm_v, const WinBwdArgs& a, const int kt, const int list,
                                            const int share, const int shares, float* part) {
  using S = WinDkvSmem<D>;
  constexpr int kStages = S::kStages, kSBufs = S::kSBufs;
  uint8_t* smem = align_1024(smem_raw);
  uint8_t* sK = smem + S::kK;
  uint8_t* sV = smem + S::kV;
  uint8_t* sQ = smem + S::kQ;
  uint8_t* sdO = smem + S::kdO;
  float* sStat = reinterpret_cast<float*>(smem + S::kStats);   // [stage][-LSE*log2e | -delta][128 queries]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::kBars);
  // p_full like s_full, one for every S^T buffer: with two buffers the softmax warps can be done with P^T of the next tile before the
  // issuer has looked for this one's, or before a slow warp has written its part of it.
  uint64_t *kv_full = bars, *s_full = bars + 1 /* [2] */, *dp_full = bars + 3, *p_full = bars + 4 /* [2] */, *ds_full = bars + 6,
           *acc_full = bars + 7, *landed = bars + 8, *q_full = bars + 9, *q_empty = q_full + kStages;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(q_empty + kStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = a.by_kv_heads.quot(list), kvh = list - b * a.kv_heads;
  const int k0 = kt * kTile, len = a.mask.length(b);
  constexpr uint32_t kTmemCols = 512;
  constexpr uint32_t kColSt = 0, kColdPt = 128 * kSBufs, kColdK = kColdPt + 128, kColdV = kColdK + D;
  constexpr int kMmaWarp = 4 * kWinGroups, kTmaWarp = kMmaWarp + 1, kCols = kTile / kWinGroups, NL = kCols / 32;
  const int g = warp >> 2, r = tid & 127;

  // the query tiles [t0, t0 + per_head) of every head of the group; full: those within [full_first, full_last)
  int first = 0, last = 0, full_first = 0, full_last = 0, t0 = 0, per_head = 0, from = 0, n_tiles = 0;
  if (k0 < len) {
    const int k_last = min(k0 + kTile, len) - 1;
    int x, y;
    a.mask.queries_of(k0, len, first, last);
    a.mask.queries_of(k_last, len, full_first, y);
    if (y > last) last = y;
    full_last = len;
    if (k_last >= a.mask.sink) a.mask.queries_of(max(k0, a.mask.sink), len, x, full_last);
    t0 = first / kTile;
    per_head = (last - 1) / kTile + 1 - t0;
    // this CTA's share of the list of (head, query tile)
    const int all = per_head * a.group;
    n_tiles = all;
    if (shares > 1) {
      from = static_cast<int>(static_cast<long long>(all) * share / shares);
      n_tiles = static_cast<int>(static_cast<long long>(all) * (share + 1) / shares) - from;
    }
  }
  if (n_tiles == 0) {   // the same for the whole CTA
    dependency_wait();
    if (warp < kMmaWarp) {
      if (part != nullptr) {
        for (int i = tid; i < 2 * kTile * D / 4; i += 32 * kMmaWarp) reinterpret_cast<float4*>(part)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      } else if (g < 2) {
        const QuadRows dk_rows = quad_rows(a.dk, b, kvh, a.mask.n, a.kv_heads, D, k0 + r), dv_rows = quad_rows(a.dv, b, kvh, a.mask.n, a.kv_heads, D, k0 + r);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          uint4 zero[4] = {};
          store_quad_rows(zero, dk_rows, g * (D / 2) + c * 32, lane);
          store_quad_rows(zero, dv_rows, g * (D / 2) + c * 32, lane);
        }
      }
    }
    return;
  }

  if (tid < 9 + 2 * kStages) {
    // q_full: a stage's bytes and the constants of its queries; p_full, ds_full: one arrival per warp
    mbar_init(bars + tid, tid >= 9 && tid < 9 + kStages ? 2 : tid >= 4 && tid <= 6 ? kMmaWarp : 1);
    fence_mbar_init();
  }
  if (tid == 0) *abort_flag = 0;
  fence_proxy_async_smem();
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_holder;
  bool redo = false;

  if (warp == kTmaWarp) {
    if (lane == 0) {
      mbar_arrive_expect_tx(kv_full, 2 * TileGeom<D>::kBytes);
      tma_load_tile<D>(sK, &tm_k, kv_full, k0, kvh, b);
      tma_load_tile<D>(sV, &tm_v, kv_full, k0, kvh, b);
    }
    dependency_wait();   // delta
    const int skipped = from == 0 ? 0 : from / per_head;
    int h = kvh * a.group + skipped, qt = t0 + from - skipped * per_head, fixes = 0;
    for (int i = 0; i < n_tiles; ++i) {
      const int st = i % kStages;
      if (!mbar_wait_ok(q_empty + st, ((i / kStages) & 1) ^ 1, abort_flag)) break;   // no copies once a wait has run out
      uint8_t *q_dst = sQ + st * TileGeom<D>::kBytes, *do_dst = sdO + st * TileGeom<D>::kBytes;
      const bool straddles = qt * kTile + kTile > len && len < a.mask.n;   // rows of Q and dO behind the end are cleared: 0 * NaN
      uint64_t* bar = straddles ? landed : q_full + st;
      if (lane == 0) {
        mbar_arrive_expect_tx(bar, 2 * TileGeom<D>::kBytes);
        tma_load_tile<D>(q_dst, &tm_q, bar, qt * kTile, h, b);
        tma_load_tile<D>(do_dst, &tm_do, bar, qt * kTile, h, b);
      }
      const size_t stat_base = (static_cast<size_t>(b) * a.heads + h) * a.mask.n;
      float* stat = sStat + st * 2 * kTile;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int qi = qt * kTile + lane * 4 + e;
        stat[lane * 4 + e] = qi < len ? -a.lse[stat_base + qi] * kLog2e : -INFINITY;
        stat[kTile + lane * 4 + e] = qi < len ? -a.delta[stat_base + qi] : 0.f;
      }
      if (straddles) {
        if (!mbar_wait_ok(landed, fixes & 1, abort_flag)) break;
        ++fixes;
        zero_rows_by_warp<D>(q_dst, len - qt * kTile, lane);
        zero_rows_by_warp<D>(do_dst, len - qt * kTile, lane);
        if (lane == 0) mbar_arrive(q_full + st);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full + st);
      if (++qt == t0 + per_head) { qt = t0; ++h; }
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0) {
      auto q_tile = [&](int i) { return smem_u32(sQ + (i % kStages) * TileGeom<D>::kBytes); };
      auto do_tile = [&](int i) { return smem_u32(sdO + (i % kStages) * TileGeom<D>::kBytes); };
      // once a wait has run out no more MMAs are issued: their operands may never have been loaded
      bool ok = true;
      auto wait_q = [&](int i) {
        ok = ok && mbar_wait_spin(q_full + i % kStages, (i / kStages) & 1, abort_flag);
        tc_fence_after_sync();
      };
      // the next S^T to issue, if there is one
      int s_next = 0;
      auto issue_s = [&]() {
        if (s_next >= n_tiles) return;
        wait_q(s_next);
        if (!ok) return;
        mma_abT<D>(tmem_base + kColSt + (s_next % kSBufs) * 128, smem_u32(sK), q_tile(s_next));
        mma_commit(s_full + s_next % kSBufs);
        ++s_next;
      };
      ok = mbar_wait_spin(kv_full, 0, abort_flag);
      issue_s();
      if (ok) {
        mma_abT<D>(tmem_base + kColdPt, smem_u32(sV), do_tile(0));
        mma_commit(dp_full);
      }
      if (kSBufs > 1) issue_s();
      for (int i = 0; ok && i < n_tiles; ++i) {
        if (!mbar_wait_spin(p_full + i % kSBufs, (i / kSBufs) & 1, abort_flag)) break;
        tc_fence_after_sync();
        win_mma_groups<D>(tmem_base + kColdV, tmem_base + kColSt + (i % kSBufs) * 128, do_tile(i), i > 0);
        issue_s();   // over P^T(i), behind the products that read it (MMAs run in order)
        if (!ok || !mbar_wait_spin(ds_full, i & 1, abort_flag)) break;
        tc_fence_after_sync();
        win_mma_groups<D>(tmem_base + kColdK, tmem_base + kColdPt, q_tile(i), i > 0);
        mma_commit(q_empty + i % kStages);
        if (i + 1 < n_tiles) {
          mma_abT<D>(tmem_base + kColdPt, smem_u32(sV), do_tile(i + 1));
          mma_commit(dp_full);
        }
      }
      mma_commit(acc_full);
    }
  } else {
    const uint32_t tmem_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const float scale_log2 = a.scale * kLog2e;
    const uint64_t sc2 = f32x2(scale_log2, scale_log2);
    const int key = k0 + r;
    const bool live = key < len;
    int q_first = 0, q_last = 0;
    if (live) a.mask.queries_of(key, len, q_first, q_last);
    const bool alone = live && a.mask.one_key(key, len);   // the query of the same token sees this key alone: dS = 0, as in dQ
    int qt = from == 0 ? t0 : t0 + from % per_head;
    for (int i = 0; i < n_tiles; ++i) {
      const float* stat = sStat + (i % kStages) * 2 * kTile + g * kCols;
      const bool full = qt * kTile >= full_first && qt * kTile + kTile <= full_last;
      const int own = alone ? key - qt * kTile - g * kCols : -1;   // its column
      uint32_t see[NL];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) {
        const int base = qt * kTile + g * kCols + c2 * 32;
        see[c2] = full ? 0xffffffffu : bits_below(q_last, base) & ~bits_below(q_first, base);
      }
      if (++qt == t0 + per_head) qt = t0;
      bool ok = mbar_wait_ok(q_full + i % kStages, (i / kStages) & 1, abort_flag);
      ok = mbar_wait_ok(s_full + i % kSBufs, (i / kSBufs) & 1, abort_flag) && ok;
      if (!ok) break;
      tc_fence_after_sync();
      const uint32_t col_s = tmem_lane + kColSt + (i % kSBufs) * 128 + g * kCols;
      uint32_t s[NL][32], pt[NL][16];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) tmem_ld32(col_s + c2 * 32, s[c2]);
      tmem_wait_ld();
      uint64_t p2[NL][16];
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2)
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const uint64_t nl2 = *reinterpret_cast<const uint64_t*>(stat + c2 * 32 + c);
          const uint64_t x2 = fma2(f32x2(__uint_as_float(s[c2][c]), __uint_as_float(s[c2][c + 1])), sc2, nl2);
          float p0, p1;
          if (((c >> 1) & 7) < kDkvPolyOf8) {
            exp2_poly_pair(x2, p0, p1);
          } else {
            float x0, x1;
            f32x2_split(x2, x0, x1);
            p0 = fast_exp2(x0);
            p1 = fast_exp2(x1);
          }
          p2[c2][c >> 1] = f32x2(p0, p1);
          pt[c2][c >> 1] = pack_bf16(p0, p1);
        }
      if (!full) {
#pragma unroll
        for (int c2 = 0; c2 < NL; ++c2)
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const uint32_t keep = ((see[c2] >> c) & 1u ? 0x0000ffffu : 0u) | ((see[c2] >> (c + 1)) & 1u ? 0xffff0000u : 0u);
            pt[c2][c >> 1] &= keep;
          }
      }
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) tmem_st16(col_s + c2 * 16, pt[c2]);
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(p_full + i % kSBufs, lane);

      if (!mbar_wait_ok(dp_full, i & 1, abort_flag)) break;
      tc_fence_after_sync();
#pragma unroll
      for (int c2 = 0; c2 < NL; ++c2) {
        uint32_t dp[32], ds[16];
        tmem_ld32(tmem_lane + kColdPt + g * kCols + c2 * 32, dp);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const uint64_t nd2 = *reinterpret_cast<const uint64_t*>(stat + kTile + c2 * 32 + c);
          const uint64_t d2 = mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c]), __uint_as_float(dp[c + 1])), nd2));
          float d0, d1;
          f32x2_split(d2, d0, d1);
          ds[c >> 1] = pack_bf16(d0, d1);
        }
        if (!full) {
          uint32_t m = see[c2];
          if (own >= c2 * 32 && own < c2 * 32 + 32 && fabsf(stat[own]) < INFINITY && fabsf(stat[kTile + own]) < INFINITY)
            m &= ~(1u << (own & 31));
#pragma unroll
          for (int c = 0; c < 32; c += 2) ds[c >> 1] &= ((m >> c) & 1u ? 0x0000ffffu : 0u) | ((m >> (c + 1)) & 1u ? 0xffff0000u : 0u);
        }
        tmem_st16(tmem_lane + kColdPt + g * kCols + c2 * 16, ds);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(ds_full, lane);
    }
    mbar_wait(acc_full, 0, abort_flag);
    tc_fence_after_sync();
    if (part != nullptr) {   // [dK | dV][128][D] in fp32, for win_join_kernel
#pragma unroll
      for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          if (c % kWinGroups != g) continue;
          uint32_t x[32];
          tmem_ld32(tmem_lane + (which ? kColdV : kColdK) + c * 32, x);
          tmem_wait_ld();
          float4* dst = reinterpret_cast<float4*>(part + (which * kTile + r) * D + c * 32);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            dst[e / 4] = make_float4(__uint_as_float(x[e]), __uint_as_float(x[e + 1]), __uint_as_float(x[e + 2]), __uint_as_float(x[e + 3]));
        }
    } else {
      const QuadRows dk_rows = quad_rows(a.dk, b, kvh, a.mask.n, a.kv_heads, D, key), dv_rows = quad_rows(a.dv, b, kvh, a.mask.n, a.kv_heads, D, key);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        if (c % kWinGroups != g) continue;
        redo = !win_store_row32(tmem_lane + kColdK + c * 32, a.scale, live, dk_rows, c * 32, lane) || redo;
        redo = !win_store_row32(tmem_lane + kColdV + c * 32, 1.f, live, dv_rows, c * 32, lane) || redo;
      }
    }
  }

  settle_after_abort(abort_flag);
  tc_fence_before_sync();
  if (__syncthreads_or(redo) && !*abort_flag) win_careful_dkv<D>(a, kt, kvh, b, warp, lane, 0, kTile);
  if (warp == kMmaWarp) tmem_dealloc(tmem_base, kTmemCols);
}

// Joins the parts of the sinks' key tiles, in their order; rows whose sums are not finite are done again by the formula.  grid.x: (key
// tile, list), grid.y: kJoinRows rows of it.
constexpr int kJoinRows = 8;
template <int D>
__global__ void __launch_bounds__(kWinBwdThreads) win_join_kernel(const WinBwdArgs a) {
  dependency_wait();
  const int i = blockIdx.x, kt = i / a.kv_lists, list = i - kt * a.kv_lists, b = list / a.kv_heads, kvh = list - b * a.kv_heads;
  const int len = a.mask.length(b), row0 = blockIdx.y * kJoinRows;
  constexpr int kVecs = kJoinRows * D / 4;           // of dK, and as many of dV
  const float4* parts = reinterpret_cast<const float4*>(a.parts) + static_cast<size_t>(i) * a.shares * (2 * kTile * D / 4) + row0 * (D / 4);
  bool redo = false;
  for (int x = threadIdx.x; x < 2 * kVecs; x += kWinBwdThreads) {
    const int which = x / kVecs, in = x - which * kVecs;
    const float4* src = parts + which * (kTile * D / 4) + in;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < a.shares; ++p) {
      const float4 v = src[static_cast<size_t>(p) * (2 * kTile * D / 4)];
      sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    const int key = kt * kTile + row0 + in / (D / 4), col = in % (D / 4) * 4;
    if (key >= a.mask.n) continue;
    const bool live = key < len;
    const float m = which ? 1.f : a.scale;
    const float chk = sum.x * m * 0.f + sum.y * m * 0.f + sum.z * m * 0.f + sum.w * m * 0.f;
    redo = redo || (live && !(chk == 0.f));
    const uint2 out = live ? make_uint2(pack_bf16(sum.x * m, sum.y * m), pack_bf16(sum.z * m, sum.w * m)) : make_uint2(0u, 0u);
    *reinterpret_cast<uint2*>((which ? a.dv : a.dk) + ((static_cast<size_t>(b) * a.mask.n + key) * a.kv_heads + kvh) * D + col) = out;
  }
  if (__syncthreads_or(redo)) win_careful_dkv<D>(a, kt, kvh, b, threadIdx.x >> 5, threadIdx.x & 31, row0, row0 + kJoinRows);
}

template <int D>
__global__ void __launch_bounds__(kWinBwdThreads, 1)
window_attn_bwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do,
                       const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const __grid_constant__ WinBwdArgs a) {
  extern __shared__ uint8_t smem_raw[];
  // key tiles forwards (the earlier ones are seen by more queries), then query tiles backwards (the later ones see more keys)
  const int front = a.front * a.kv_lists * a.shares;   // CTAs of the sinks' key tiles, `shares` to a tile
  const int behind = a.kv_lists * (a.tiles - a.front);
  int i = blockIdx.x;
  if (i < front) {
    int x = i, share = 0, kt = 0;
    if (a.shares > 1) { x = i / a.shares; share = i - x * a.shares; }
    if (a.front > 1) kt = x / a.kv_lists;
    const int list = x - kt * a.kv_lists;
    win_bwd_dkv<D>(smem_raw, tm_q, tm_do, tm_k, tm_v, a, kt, list, share, a.shares,
                   a.shares > 1 ? a.parts + static_cast<size_t>(i) * (2 * kTile * D) : nullptr);
  } else if ((i -= front) < behind) {
    int tile, list;
    a.k_order.place(i, tile, list);
    win_bwd_dkv<D>(smem_raw, tm_q, tm_do, tm_k, tm_v, a, a.front + tile, list, 0, 1, nullptr);
  } else {
    int tile, list;
    a.q_order.place(i - behind, tile, list);
    win_bwd_dq<D>(smem_raw, tm_k, tm_v, tm_do, a, a.tiles - 1 - tile, list);
  }
}
template <int D> constexpr int window_bwd_smem() {
  return DqSmem<D>::kTotal > WinDkvSmem<D>::kTotal ? DqSmem<D>::kTotal : WinDkvSmem<D>::kTotal;
}

}  // namespace astro
