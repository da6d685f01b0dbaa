// Backward of attention over lists of key blocks, the cached context detached.
//   dQ kernel     a query tile stationary, over the key tiles of its list:  dQ = scale * sum dS K
//   dK/dV kernel  a chunk key block stationary, over the query tiles whose lists name it (sparse_bwd_prep_kernel turns the
//                 lists around): dV = sum P^T dO, dK = scale * sum dS^T Q
// with P = exp(S - LSE), dS = P o (dP - delta), as in the dense kernels, whose tensor-memory layouts, operand forms and
// hand-offs these two have: see there.  No atomics touch a sum: the counts that turn the lists around are whole numbers
// and every accumulator belongs to one CTA, so results do not depend on the order of anything.
// Precision: bf16 products, fp32 sums; P and dS are rounded to bf16 (half a step, 2^-8 of each term at most) as operands
// of the second products.
// Bound: the tensor pipe and its hand-offs, as in the dense kernels: a key tile of dQ takes 2140 clocks (MMAs 1536), a query tile
// of dK/dV 2730 (2048); setting up and finishing a CTA adds 7 % and, with 9 query tiles per chunk block, 21 %.  Clip shape (batch 2,
// 64 of 273 blocks): 677 us in one launch, 674 in two with a gap between them; preparation 13.7 us.
#pragma once
#include "attn_bwd.cuh"
#include "sparse_common.cuh"

namespace astro {

// What both kernels need, in one launch.
//   delta[b][h][i] = dO_i . O_i, fp32: D/8 lanes per row, 16 bytes of both tensors each; bandwidth
//   counts[b][h][chunk block][query tile] = times that the query tile's list names the block: a warp per list and 1024 chunk
//   blocks counts them in shared memory and writes every count, zeros included
// The first `count_blocks` thread blocks count, the others take 256 * kDeltaRows * 8 / D rows each.
constexpr int kPrepThreads = 256, kDeltaRows = 2, kCountSpan = 1024;

struct SparsePrepArgs {
  const __nv_bfloat16 *o, *d_o;
  const int* blocks;
  float* delta;
  int* counts;
  long long rows;    // batch * n_q * heads
  long long lists;   // batch * heads * q_tiles
  long long count_blocks;
  int heads, n_q, q_tiles, n_select, ctx_blocks, chunk_blocks, spans;
};

template <int D>
__global__ void __launch_bounds__(kPrepThreads)
sparse_bwd_prep_kernel(const SparsePrepArgs a) {
  __shared__ int hist[kPrepThreads / 32][kCountSpan];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  dependents_may_start();
  if (blockIdx.x < a.count_blocks) {
    const long long job = static_cast<long long>(blockIdx.x) * (kPrepThreads / 32) + warp;   // (list, span)
    if (job >= a.lists * a.spans) return;
    const long long list = job / a.spans;
    const int first = static_cast<int>(job - list * a.spans) * kCountSpan, n = min(kCountSpan, a.chunk_blocks - first);
    int* own = hist[warp];
    for (int i = lane; i < n; i += 32) own[i] = 0;
    __syncwarp();
    const int* ids = a.blocks + list * a.n_select;
    for (int i = lane; i < a.n_select; i += 32) {
      const int id = ids[i];
      if (id >= a.ctx_blocks && id - a.ctx_blocks >= first && id - a.ctx_blocks < first + n)
        atomicAdd(own + (id - a.ctx_blocks - first), 1);
    }
    __syncwarp();
    const long long bh = list / a.q_tiles, qt = list - bh * a.q_tiles;
    for (int i = lane; i < n; i += 32) a.counts[(bh * a.chunk_blocks + first + i) * a.q_tiles + qt] = own[i];
    return;
  }
  constexpr int kLanes = D / 8, kPerPass = kPrepThreads / kLanes;
  const int part = threadIdx.x % kLanes;
  const long long row0 = (static_cast<long long>(blockIdx.x) - a.count_blocks) * (kPerPass * kDeltaRows) + threadIdx.x / kLanes;
  uint4 x[kDeltaRows], y[kDeltaRows];
#pragma unroll
  for (int u = 0; u < kDeltaRows; ++u) {
    const long long row = row0 + u * kPerPass;
    if (row < a.rows) {
      x[u] = *reinterpret_cast<const uint4*>(a.o + row * D + part * 8);
      y[u] = *reinterpret_cast<const uint4*>(a.d_o + row * D + part * 8);
    } else {
      x[u] = y[u] = make_uint4(0, 0, 0, 0);
    }
  }
#pragma unroll
  for (int u = 0; u < kDeltaRows; ++u) {
    const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162*>(&x[u]), *q = reinterpret_cast<const __nv_bfloat162*>(&y[u]);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __bfloat1622float2(p[e]), g = __bfloat1622float2(q[e]);
      sum = fmaf(f.x, g.x, sum);
      sum = fmaf(f.y, g.y, sum);
    }
#pragma unroll
    for (int s = kLanes / 2; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    const long long row = row0 + u * kPerPass;
    if (part == 0 && row < a.rows) {
      if (a.rows <= 0x7fffffffLL) {   // divisions of 32 bits where they do (15.1 us against 16.7)
        const unsigned x = static_cast<unsigned>(row), bi = x / a.heads, b = bi / a.n_q;
        a.delta[(static_cast<size_t>(b) * a.heads + (x - bi * a.heads)) * a.n_q + (bi - b * a.n_q)] = sum;
      } else {
        const long long bi = row / a.heads, b = bi / a.n_q;
        a.delta[(b * a.heads + (row - bi * a.heads)) * a.n_q + (bi - b * a.n_q)] = sum;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------ dQ
struct SparseBwdArgs {
  const __nv_bfloat16* q;
  const int* blocks;
  const float *lse, *delta;
  __nv_bfloat16* dq;
  int batch, heads, n_q, q_tiles, n_select, cache_shared;
  float scale;
};

// A warp of its own follows the list and describes the tiles to come in a ring (listed: written; unlisted: everyone has
// read it).  The rest is the dense dQ kernel with `last` read out of the descriptors.
constexpr int kSparseBwdThreads = kDqSoftmaxThreads + 96;   // MMA, loads, list

template <int D> struct SdqSmem {
  static constexpr int kBars = DqSmem<D>::kBars;
  static constexpr int kDesc = kBars + 40 * 8;
  static constexpr int kSource = kDesc + kSpDescs * static_cast<int>(sizeof(TileDesc));
  static constexpr int kTotal = kSource + kSpDescs * static_cast<int>(sizeof(TileSource)) + 1024;
};

template <int D>
__device__ __forceinline__ void sparse_bwd_dq(uint8_t* smem_raw, const SparseMaps& maps, const CUtensorMap& tm_do,
                                              const SparseGeom& geom, const SparseBwdArgs& a, const int qt, const int h, const int b) {
  uint8_t* smem = align_1024(smem_raw);
  uint8_t* sdO = smem + DqSmem<D>::kdO;
  uint8_t* sK = smem + DqSmem<D>::kK;
  uint8_t* sV = smem + DqSmem<D>::kV;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + SdqSmem<D>::kBars);
  uint64_t *kv0_full = bars, *qt_full = bars + 1, *rs = bars + 2, *rb = bars + 6, *s_full = bars + 10, *b_done = bars + 11,
           *dq_full = bars + 13, *listed = bars + 14, *unlisted = bars + 14 + kSpDescs;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bars + 14 + 2 * kSpDescs);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  TileDesc* desc = reinterpret_cast<TileDesc*>(smem + SdqSmem<D>::kDesc);
  TileSource* source = reinterpret_cast<TileSource*>(smem + SdqSmem<D>::kSource);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int q0 = qt * kTile;
  const int bx = a.cache_shared ? 0 : b;
  constexpr uint32_t kTmemCols = 512;
  constexpr uint32_t kColS = 0, kColdP = 128, kColdS = 256, kColQ = 320, kColdQ = 384;
  constexpr int kMmaWarp = 4 * kDqGroups, kTmaWarp = kMmaWarp + 1, kListWarp = kMmaWarp + 2;

  // the list's first entries are on their way while barriers and tensor memory are set up
  const int* list = a.blocks + ((static_cast<long long>(b) * a.heads + h) * a.q_tiles + qt) * a.n_select;
  int first_entries = -1;
  if (warp == kListWarp) first_entries = ListWalker::first_entries(list, a.n_select, lane);
  if (warp == kTmaWarp && lane == 0) {
    tma_prefetch_desc(&maps.kx); tma_prefetch_desc(&maps.vx); tma_prefetch_desc(&maps.kc); tma_prefetch_desc(&maps.vc);
    tma_prefetch_desc(&tm_do);
  }
  if (tid < 14 + 2 * kSpDescs) {   // every barrier is set up by a thread of its own
    // qt_full: one arrival per warp and 64 elements; rs, rb: bytes and warps; unlisted: the list's readers
    mbar_init(bars + tid, tid == 1 ? 4 * (D / 64) : tid >= 2 && tid < 10 ? 1 + 4 * kDqGroups : tid < 14 + kSpDescs ? 1 : 4 * kDqGroups + 2);
    fence_mbar_init();
  }
  if (tid == 0) *abort_flag = 0;
  zero_uncovered_rows<D>(sK, kDqKStages, geom, tid, kSparseBwdThreads);
  zero_uncovered_rows<D>(sV, kDqVStages, geom, tid, kSparseBwdThreads);
  fence_proxy_async_smem();
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_holder;
  dependents_may_start();
  // a descriptor's reading, and its return (a warp's readers return it together)
  auto await_listed = [&](int j) { return mbar_wait_spin(listed + j % kSpDescs, (j / kSpDescs) & 1, abort_flag); };

  if (warp == kListWarp) {
    ListWalker w;
    w.open(geom, list, a.n_select, lane, first_entries);
    for (int j = 0;; ++j) {
      if (!mbar_wait_ok(unlisted + j % kSpDescs, ((j / kSpDescs) & 1) ^ 1, abort_flag)) break;
      uint32_t valid;
      const bool last = next_tile(geom, w, h, b, bx, source + j % kSpDescs, valid);
      if (lane == 0) {
        desc[j % kSpDescs].valid = valid;
        desc[j % kSpDescs].flags = kTileThere | (last ? kTileLast : 0u);
        mbar_arrive(listed + j % kSpDescs);
      }
      if (last) break;
    }
  } else if (warp == kTmaWarp) {
    if (lane == 0) {
      const uint32_t bytes = sparse_tile_bytes<D>(geom);
      auto load_kv = [&](int t, uint64_t* k_bar, uint64_t* v_bar) {
        load_sparse_tile<D>(sK + (t % kDqKStages) * TileGeom<D>::kBytes, &maps.kx, &maps.kc, k_bar, source + t % kSpDescs, geom);
        load_sparse_tile<D>(sV + (t % kDqVStages) * TileGeom<D>::kBytes, &maps.vx, &maps.vc, v_bar, source + t % kSpDescs, geom);
      };
      bool last = false;
      if (await_listed(0)) {
        mbar_arrive_expect_tx(kv0_full, TileGeom<D>::kBytes + 2 * bytes);
        tma_load_tile<D>(sdO, &tm_do, kv0_full, q0, h, b);
        load_kv(0, kv0_full, kv0_full);
        last = reinterpret_cast<volatile TileDesc*>(desc)->flags & kTileLast;
        mbar_arrive(unlisted);
        for (int t = 1;; ++t) {
          if (!last && !await_listed(t)) break;
          // commit t-1 of b_done: dQ(t-3) and dP(t-2) are done, the K stage and the V stage of tile t are free
          if (t >= 2 && !mbar_wait_spin(b_done + ((t - 1) & 1), ((t - 2) >> 1) & 1, abort_flag)) break;
          if (last) {
            mbar_arrive(rb + (t - 1) % 4);   // the last tile's burst waits for no bytes (its rs is never awaited)
            break;
          }
          mbar_arrive_expect_tx(rs + (t - 1) % 4, bytes);
          mbar_arrive_expect_tx(rb + (t - 1) % 4, bytes);
          load_kv(t, rs + (t - 1) % 4, rb + (t - 1) % 4);
          last = reinterpret_cast<volatile TileDesc*>(desc + t % kSpDescs)->flags & kTileLast;
          mbar_arrive(unlisted + t % kSpDescs);
        }
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
      auto last_tile = [&](int j, bool& ok) {
        ok = await_listed(j) && ok;
        const bool last = reinterpret_cast<volatile TileDesc*>(desc + j % kSpDescs)->flags & kTileLast;
        mbar_arrive(unlisted + j % kSpDescs);
        return last;
      };
      bool ok = mbar_wait_spin(qt_full, 0, abort_flag);
      ok = mbar_wait_spin(kv0_full, 0, abort_flag) && ok;
      tc_fence_after_sync();
      issue_s(0);
      issue_dp(0);
      mma_commit(b_done + 1);                       // commit 1
      bool last = last_tile(0, ok);
      for (int j = 0; ok; ++j) {
        if (!last) {
          ok = mbar_wait_spin(rs + j % 4, (j / 4) & 1, abort_flag);
          tc_fence_after_sync();
          issue_s(j + 1);
        }
        ok = mbar_wait_spin(rb + j % 4, (j / 4) & 1, abort_flag) && ok;
        tc_fence_after_sync();
        if (!last) issue_dp(j + 1);
        mma_pb<D, kTile>(tmem_base + kColdQ, tmem_base + kColdS, smem_u32(sK + (j % kDqKStages) * TileGeom<D>::kBytes), j > 0);
        mma_commit(b_done + (j & 1));                 // commit j + 2
        if (last) break;
        last = last_tile(j + 1, ok);
      }
      mma_commit(dq_full);
    }
  } else {
    const int g = warp >> 2;
    const int r = tid & 127;
    const uint32_t tmem_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const int row = q0 + r;
    const bool in_range = row < a.n_q;
    const size_t stat_idx = (static_cast<size_t>(b) * a.heads + h) * a.n_q + (in_range ? row : 0);
    dependency_wait();   // delta
    const float lse2 = in_range ? a.lse[stat_idx] * kLog2e : 0.f;
    const float delta_r = in_range ? a.delta[stat_idx] : 0.f;
    const float scale_log2 = a.scale * kLog2e;
    const uint64_t sc2 = f32x2(scale_log2, scale_log2), nl2 = f32x2(-lse2, -lse2), nd2 = f32x2(-delta_r, -delta_r);
    const bool idle = q0 + (warp & 3) * 32 >= a.n_q;   // no query among the warp's rows: it only keeps the hand-offs going
    if (g * 64 < D) {   // Q row -> tensor memory: group g writes elements [64g, 64g+64) of its row as 32 packed columns
      uint32_t qr[32];
      const QuadRows q_rows = quad_rows(a.q, b, h, a.n_q, a.heads, D, row);
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
    static_assert(kDqCols == 64, "two 32-key pieces per thread and tile");
    for (int j = 0;; ++j) {
      bool ok = await_listed(j);
      const uint32_t flags = reinterpret_cast<volatile TileDesc*>(desc + j % kSpDescs)->flags;
      const uint32_t valid = reinterpret_cast<volatile TileDesc*>(desc + j % kSpDescs)->valid >> (16 * g);   // two bytes
      __syncwarp();
      if (lane == 0) mbar_arrive(unlisted + j % kSpDescs);
      ok = mbar_wait_ok(s_full, j & 1, abort_flag) && ok;
      tc_fence_after_sync();
      if (idle) {   // rows of an MMA do not mix: what dS holds here ends in rows of dQ that nobody stores
        warp_arrive(rs + j % 4, lane);
        ok = mbar_wait_ok(b_done + ((j + 1) & 1), (j >> 1) & 1, abort_flag) && ok;
        warp_arrive(rb + j % 4, lane);
        if ((flags & kTileLast) || !__all_sync(0xffffffffu, ok)) break;
        continue;
      }
      uint32_t s[2][32];
      tmem_ld32(tmem_lane + kColS + g * kDqCols, s[0]);
      tmem_ld32(tmem_lane + kColS + g * kDqCols + 32, s[1]);
      tmem_wait_ld();
      tc_fence_before_sync();
      warp_arrive(rs + j % 4, lane);
      uint64_t p2[2][16];
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2)
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          float x0, x1;
          f32x2_split(fma2(f32x2(__uint_as_float(s[c2][c]), __uint_as_float(s[c2][c + 1])), sc2, nl2), x0, x1);
          p2[c2][c >> 1] = f32x2(fast_exp2(x0), fast_exp2(x1));
        }
      // commit j+1 of b_done: dP(j) is there, and dQ(j-1) has consumed the one dS buffer
      ok = mbar_wait_ok(b_done + ((j + 1) & 1), (j >> 1) & 1, abort_flag) && ok;
      tc_fence_after_sync();
      uint32_t dp[2][32], ds[2][16];
      tmem_ld32(tmem_lane + kColdP + g * kDqCols, dp[0]);
      tmem_ld32(tmem_lane + kColdP + g * kDqCols + 32, dp[1]);
      tmem_wait_ld();
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        const int v = (valid >> (8 * c2)) & 0xff;
        if (v >= 32) {
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float d0, d1;
            f32x2_split(mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c2][c]), __uint_as_float(dp[c2][c + 1])), nd2)), d0, d1);
            ds[c2][c >> 1] = pack_bf16(d0, d1);
          }
        } else {   // rows that are no key: P can be anything there (exp(-LSE) of an empty row is infinite), dS is 0
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            float d0, d1;
            f32x2_split(mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c2][c]), __uint_as_float(dp[c2][c + 1])), nd2)), d0, d1);
            ds[c2][c >> 1] = pack_bf16(c < v ? d0 : 0.f, c + 1 < v ? d1 : 0.f);
          }
        }
        tmem_st16(tmem_lane + kColdS + g * (kDqCols / 2) + c2 * 16, ds[c2]);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(rb + j % 4, lane);   // dS(j) stored; dP(j) was read before it, so its buffer is free as well
      if ((flags & kTileLast) || !__all_sync(0xffffffffu, ok)) break;
    }
    mbar_wait(dq_full, 0, abort_flag);
    tc_fence_after_sync();
    store_rows_from_tmem<D / 2>(tmem_lane + kColdQ + g * (D / 2), a.scale, quad_rows(a.dq, b, h, a.n_q, a.heads, D, row),
                                g * (D / 2), lane);
  }

  settle_after_abort(abort_flag);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(tmem_base, kTmemCols);
}

// ------------------------------------------------------------------------------------------ dK, dV
struct SparseDkvArgs {
  const int* counts;     // [B][H][chunk blocks][q_tiles]
  __nv_bfloat16 *dk, *dv;
  const float *lse, *delta;
  int heads, n_q, n_kc, q_tiles, block, chunk_blocks;
  float scale;
};

// One CTA per chunk key block: the dense dK/dV kernel with the query tiles that name the block instead of all.  The producer warp
// walks along the block's counts, 32 query tiles at a time, and takes a tile as often as it is counted.  A block that no
// list names gets zeros.  Blocks of fewer than 128 tokens leave rows of the key tile empty (zeros in shared memory): blocks of 64
// cost twice the work, which a tile of several blocks could save only for query tiles that name all of them.
template <int D>
__device__ __forceinline__ void sparse_bwd_dkv(uint8_t* smem_raw, const CUtensorMap& tm_q, const CUtensorMap& tm_do,
                                               const CUtensorMap& tm_kc, const CUtensorMap& tm_vc, const SparseDkvArgs& a,
                                               const int cb, const int h, const int b) {
  uint8_t* smem = align_1024(smem_raw);
  uint8_t* sK = smem + DkvSmem<D>::kK;
  uint8_t* sV = smem + DkvSmem<D>::kV;
  uint8_t* sQ = smem + DkvSmem<D>::kQ;
  uint8_t* sdO = smem + DkvSmem<D>::kdO;
  float* sStat = reinterpret_cast<float*>(smem + DkvSmem<D>::kStats);   // [stage][-LSE*log2e | -delta][128 queries]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + DkvSmem<D>::kBars);
  uint64_t* kv_full = bars;
  uint64_t* q_full = bars + 1;
  uint64_t* q_empty = q_full + kDkvStages;
  uint64_t* s_full = q_empty + kDkvStages;
  uint64_t* dp_full = s_full + 1;
  uint64_t* p_full = dp_full + 1;
  uint64_t* ds_full = p_full + 1;
  uint64_t* acc_full = ds_full + 1;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(acc_full + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  volatile int* tiles_holder = reinterpret_cast<volatile int*>(tmem_holder + 2);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int k0 = cb * a.block, keys = min(a.block, a.n_kc - k0);
  constexpr uint32_t kTmemCols = 512;
  constexpr uint32_t kColSt = 0, kColdPt = 128, kColdK = 256, kColdV = 384;
  constexpr int kMmaWarp = 8, kTmaWarp = 9;
  constexpr int kHalfBytes = 64 * 128;
  const int* counts = a.counts + ((static_cast<long long>(b) * a.heads + h) * a.chunk_blocks + cb) * a.q_tiles;

  if (tid == 0) {
    mbar_init(kv_full, 1);
    for (int i = 0; i < kDkvStages; ++i) { mbar_init(q_full + i, 2); mbar_init(q_empty + i, 1); }
    mbar_init(s_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(p_full, 8);    // one arrival per warp
    mbar_init(ds_full, 8);
    mbar_init(acc_full, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  SparseGeom geom;
  geom.kb.block = a.block;
  geom.pad = kTile;
  geom.per_tile = 1;
  zero_uncovered_rows<D>(sK, 2, geom, tid, kSparseBwdThreads);   // K and V of the block follow each other
  fence_proxy_async_smem();
  dependency_wait();   // counts and delta
  if (warp == kTmaWarp) {
    int n = 0;
    for (int t = lane; t < a.q_tiles; t += 32) n += counts[t];
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) *tiles_holder = n;
  }
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_holder;
  const int n_tiles = *tiles_holder;

  if (warp == kTmaWarp) {
    const size_t stat_base = (static_cast<size_t>(b) * a.heads + h) * a.n_q;
    if (lane == 0 && n_tiles > 0) {
      mbar_arrive_expect_tx(kv_full, 2 * a.block * 128 * TileGeom<D>::kBlocks);
#pragma unroll
      for (int blk = 0; blk < TileGeom<D>::kBlocks; ++blk) {
        tma_load_5d(sK + blk * TileGeom<D>::kBlockBytes, &tm_kc, kv_full, blk * 64, k0, 0, h, b);
        tma_load_5d(sV + blk * TileGeom<D>::kBlockBytes, &tm_vc, kv_full, blk * 64, k0, 0, h, b);
      }
    }
    int base = -32, left = 0, times = 0, qt = 0;   // 32 counts in the lanes; the tile at hand and how often it is still due
    uint32_t mask = 0;
    for (int i = 0; i < n_tiles; ++i) {
      if (times == 0) {
        while (mask == 0 && base + 32 < a.q_tiles) {   // the counts behind `base` add up to the tiles still due
          base += 32;
          left = base + lane < a.q_tiles ? counts[base + lane] : 0;
          mask = __ballot_sync(0xffffffffu, left > 0);
        }
        const int from = (__ffs(mask) - 1) & 31;
        mask &= mask - 1;
        qt = base + from;
        times = __shfl_sync(0xffffffffu, left, from);
      }
      --times;
      const int st = i % kDkvStages;
      const bool go = mbar_wait_ok(q_empty + st, ((i / kDkvStages) & 1) ^ 1, abort_flag);
      if (!go) break;   // no copies once a wait has run out
      if (lane == 0) {
        mbar_arrive_expect_tx(q_full + st, 2 * TileGeom<D>::kBytes);
        tma_load_tile<D>(sQ + st * TileGeom<D>::kBytes, &tm_q, q_full + st, qt * kTile, h, b);
        tma_load_tile<D>(sdO + st * TileGeom<D>::kBytes, &tm_do, q_full + st, qt * kTile, h, b);
      }
      float* stat = sStat + st * 2 * kTile;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int qi = qt * kTile + lane * 4 + e;
        stat[lane * 4 + e] = qi < a.n_q ? -a.lse[stat_base + qi] * kLog2e : -INFINITY;   // P = 0 for rows past n_q
        stat[kTile + lane * 4 + e] = qi < a.n_q ? -a.delta[stat_base + qi] : 0.f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full + st);
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0 && n_tiles > 0) {
      auto q_tile = [&](int i) { return smem_u32(sQ + (i % kDkvStages) * TileGeom<D>::kBytes); };
      auto do_tile = [&](int i) { return smem_u32(sdO + (i % kDkvStages) * TileGeom<D>::kBytes); };
      // once a wait has run out no more MMAs are issued: their operands may never have been loaded
      bool ok = true;
      auto wait_q = [&](int i) {
        ok = ok && mbar_wait_spin(q_full + i % kDkvStages, (i / kDkvStages) & 1, abort_flag);
        tc_fence_after_sync();
      };
      ok = mbar_wait_spin(kv_full, 0, abort_flag);
      wait_q(0);
      if (ok) {
        mma_abT<D>(tmem_base + kColSt, smem_u32(sK), q_tile(0));
        mma_commit(s_full);
        mma_abT<D>(tmem_base + kColdPt, smem_u32(sV), do_tile(0));
        mma_commit(dp_full);
      }
      for (int i = 0; ok && i < n_tiles; ++i) {
        if (!mbar_wait_spin(p_full, i & 1, abort_flag)) break;
        tc_fence_after_sync();
        mma_pb<D, 64>(tmem_base + kColdV, tmem_base + kColSt, do_tile(i), i > 0);
        mma_pb<D, 64>(tmem_base + kColdV, tmem_base + kColSt + 64, do_tile(i) + kHalfBytes, true);
        if (i + 1 < n_tiles) {
          wait_q(i + 1);
          if (!ok) break;
          mma_abT<D>(tmem_base + kColSt, smem_u32(sK), q_tile(i + 1));
          mma_commit(s_full);
        }
        if (!mbar_wait_spin(ds_full, i & 1, abort_flag)) break;
        tc_fence_after_sync();
        mma_pb<D, 64>(tmem_base + kColdK, tmem_base + kColdPt, q_tile(i), i > 0);
        mma_pb<D, 64>(tmem_base + kColdK, tmem_base + kColdPt + 64, q_tile(i) + kHalfBytes, true);
        mma_commit(q_empty + i % kDkvStages);
        if (i + 1 < n_tiles) {
          mma_abT<D>(tmem_base + kColdPt, smem_u32(sV), do_tile(i + 1));
          mma_commit(dp_full);
        }
      }
      mma_commit(acc_full);
    }
  } else if (warp < kMmaWarp) {
    const int g = warp >> 2;
    const int r = tid & 127;  // key row inside the tile = TMEM lane
    const uint32_t tmem_lane = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const float scale_log2 = a.scale * kLog2e;
    const uint64_t sc2 = f32x2(scale_log2, scale_log2);
    for (int i = 0; i < n_tiles; ++i) {
      const float* stat = sStat + (i % kDkvStages) * 2 * kTile + g * 64;
      bool ok = mbar_wait_ok(q_full + i % kDkvStages, (i / kDkvStages) & 1, abort_flag);
      ok = mbar_wait_ok(s_full, i & 1, abort_flag) && ok;
      if (!ok) break;
      tc_fence_after_sync();
      uint32_t s[2][32], pt[32];
      tmem_ld32(tmem_lane + kColSt + g * 64, s[0]);
      tmem_ld32(tmem_lane + kColSt + g * 64 + 32, s[1]);
      tmem_wait_ld();
      uint64_t p2[2][16];
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2)
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
          pt[c2 * 16 + (c >> 1)] = pack_bf16(p0, p1);
        }
      tmem_st32(tmem_lane + kColSt + g * 64, pt);
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(p_full, lane);

      if (!mbar_wait_ok(dp_full, i & 1, abort_flag)) break;
      tc_fence_after_sync();
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        uint32_t dp[32], ds[16];
        tmem_ld32(tmem_lane + kColdPt + g * 64 + c2 * 32, dp);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          const uint64_t nd2 = *reinterpret_cast<const uint64_t*>(stat + kTile + c2 * 32 + c);
          const uint64_t d2 = mul2(p2[c2][c >> 1], add2(f32x2(__uint_as_float(dp[c]), __uint_as_float(dp[c + 1])), nd2));
          float d0, d1;
          f32x2_split(d2, d0, d1);
          ds[c >> 1] = pack_bf16(d0, d1);
        }
        tmem_st16(tmem_lane + kColdPt + g * 64 + c2 * 16, ds);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive(ds_full, lane);
    }
    // the rows of a quad that are keys of this block
    auto rows_of = [&](__nv_bfloat16* base) {
      QuadRows q;
      const int first = r & ~3;
      q.stride = static_cast<size_t>(a.heads) * D;
      q.first = base + (static_cast<size_t>(b) * a.n_kc + k0 + first) * q.stride + static_cast<size_t>(h) * D;
      q.valid = keys - first;
      return q;
    };
    if (n_tiles > 0) {
      mbar_wait(acc_full, 0, abort_flag);
      tc_fence_after_sync();
      store_rows_from_tmem<D / 2>(tmem_lane + kColdK + g * (D / 2), a.scale, rows_of(a.dk), g * (D / 2), lane);
      store_rows_from_tmem<D / 2>(tmem_lane + kColdV + g * (D / 2), 1.f, rows_of(a.dv), g * (D / 2), lane);
    } else {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        uint4 zero[4] = {};
        store_quad_rows(zero, rows_of(a.dk), g * (D / 2) + c * 32, lane);
        store_quad_rows(zero, rows_of(a.dv), g * (D / 2) + c * 32, lane);
      }
    }
  }

  settle_after_abort(abort_flag);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(tmem_base, kTmemCols);
}

// Both in one launch: the first CTAs take the query tiles (the longer job), the others the chunk blocks.  Neither needs the
// other, and one launch leaves no SM idle between them.
template <int D>
__global__ void __launch_bounds__(kSparseBwdThreads, 1)
sparse_attn_bwd_kernel(const __grid_constant__ SparseMaps maps, const __grid_constant__ CUtensorMap tm_q,
                       const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ SparseGeom geom,
                       const __grid_constant__ SparseBwdArgs a, const __grid_constant__ SparseDkvArgs k, const int q_ctas) {
  extern __shared__ uint8_t smem_raw[];
  int i = blockIdx.x;
  if (i < q_ctas) {
    const int qt = i % a.q_tiles;
    i /= a.q_tiles;
    // with one stored prefix for every sample, the samples of a head run next to each other (see the dense kernel)
    const int inner = a.cache_shared ? a.batch : a.heads, y = i % inner, z = i / inner;
    sparse_bwd_dq<D>(smem_raw, maps, tm_do, geom, a, qt, a.cache_shared ? z : y, a.cache_shared ? y : z);
  } else {
    i -= q_ctas;
    const int cb = i % k.chunk_blocks;
    i /= k.chunk_blocks;
    sparse_bwd_dkv<D>(smem_raw, tm_q, tm_do, maps.kc, maps.vc, k, cb, i % k.heads, i / k.heads);
  }
}
template <int D> constexpr int sparse_bwd_smem() {
  return SdqSmem<D>::kTotal > DkvSmem<D>::kTotal ? SdqSmem<D>::kTotal : DkvSmem<D>::kTotal;
}

}  // namespace astro
