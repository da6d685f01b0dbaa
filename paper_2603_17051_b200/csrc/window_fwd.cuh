// Forward of attention with a sliding window and sinks over whole sequences (window_common.cuh): O and LSE.
//
// Built like the dense forward (attn_fwd.cuh): a work unit is a 128-query tile of one head of one sample; four softmax groups of 128
// threads, one thread that issues every tcgen05 MMA, a warp each for the loads of K and V, eight epilogue warps that bring Q
// and take O out; the key tiles of all the units of a CTA form one stream, S two tiles ahead of P V; one wait and one commit of the
// issuing thread per key tile.  Tensor-memory layout as there.  What differs:
//   * A unit's key tiles are those of window_common.cuh, its own (diagonal) tile first: there every query sees a key, itself,
//     so its maximum is a reference that every row has.  Only tiles that are not full pay for a mask (a bit per key and row).
//   * Units differ in length (a video's first chunk has 37 key tiles, its last 147 or more), so they are not dealt out beforehand.
//     The grid has a CTA per unit; a running CTA takes the next unit from the hardware's queue of CTAs not yet launched
//     (clusterlaunchcontrol), one unit ahead of the one it works on.  Long units come first.
//   * K and V are shared by heads / kv_heads heads; q, k and v may be strided.
//   * Keys from a sequence's length on may be anything, NaN included: their scores are masked, and V's rows are cleared in
//     shared memory where a tile straddles the end (0 * NaN would reach O).  Within a sequence an infinity or NaN in a value of a
//     tile that only some rows see would reach the others the same way: like a row sum beyond 2^100, a result that is not finite sends
//     the unit to a second pass on the ordinary cores, key by key, which is the formula and nothing else.  Slow and rare.
// Bound: as the dense forward, by the tensor pipe, the exponentials and power together: a video's 32760 tokens (blocks of 4680, a
// window of 18720, 4680 sinks, 12 heads of 128) in 2510 us, 1340 TFLOP/s of the pairs that are seen, tensor pipe 73 %.  16384 causal
// tokens, 12 heads: 637 us at head_dim 128, 528 at 64 (exponentials).  Short calls are latency: 300 tokens in 8.9 us.
// Precision: bf16 products, fp32 sums; P is rounded to bf16 for P V (half a step, 2^-8 of each weight at most), the row sum is
// taken from the fp32 values.
#pragma once
#include "attn_fwd.cuh"
#include "sparse_common.cuh"
#include "window_common.cuh"

namespace astro {

struct WinFwdArgs {
  const __nv_bfloat16 *q, *k, *v;
  WinStrides qs, ks, vs;
  __nv_bfloat16* o;        // [B, n, H, D]
  float* lse;              // [B, H, n], may be null
  WinMask mask;
  int heads, group;        // group: heads that share K and V
  Divisor by_heads, by_group;
  WinOrder order;
  float scale, scale_log2;
  int careful;             // 1: the second pass only
};

constexpr int kWinMaxUnits = 1024;                       // of one CTA; it asks no more often
constexpr int kWinThreads = 128 * kFwdGroups + 32 * (4 + kFwdEpiWarps);   // + MMA, units, K, V
constexpr int kWinBarSlots = 40;

struct WinUnitInfo {
  int id, tiles;           // id < 0: there is none
};

template <int D> struct WinFwdSmem {
  static constexpr int kK = FwdSmem<D>::kK;
  static constexpr int kV = FwdSmem<D>::kV;
  static constexpr int kMax = FwdSmem<D>::kMax;
  static constexpr int kBars = FwdSmem<D>::kBars;
  static constexpr int kHolder = kBars + kWinBarSlots * 8;                     // tensor memory's address, abort flag
  static constexpr int kAnswer = kHolder + 16;                                 // of the queue of units, 16 bytes
  static constexpr int kUnits = kAnswer + 16;
  static constexpr int kRedo = kUnits + (kWinMaxUnits + 2) * static_cast<int>(sizeof(WinUnitInfo));
  static constexpr int kTotal = kRedo + (kWinMaxUnits / 32 + 1) * 4 + 1024;
};

// Unit id -> query tile, head, sample (WinOrder, the query tiles backwards: the long ones first).
struct WinUnit {
  int qt, h, b;
  __device__ __forceinline__ WinUnit(const WinFwdArgs& a, int id) {
    int tile, list;
    a.order.place(id, tile, list);
    qt = a.order.tiles - 1 - tile;
    b = a.by_heads.quot(list);
    h = list - b * a.heads;
  }
};

// Barriers: the dense fast pass's (slots 0..22) with arrivals of whole warps, and
//   max_full[4]  the warps of a quarter have left their first-tile maxima     k_pre[2]  K of the stream's first two tiles
//   listed[4]    unit n is known (slot n % 4)                                  answer    of the queue of units
//   landed       V of a tile that straddles the end of its sequence            done[4]  unit n's products are complete (slot n % 4)
struct WinBars : FwdFastBars {
  uint64_t *max_full, *k_pre, *listed, *answer, *landed, *done;
  __device__ explicit WinBars(uint64_t* b)
      : FwdFastBars(b), max_full(b + 23), k_pre(b + 27), listed(b + 29), answer(b + 33), landed(b + 34), done(b + 35) {}
  static __device__ int arrivals(int i) {
    if (i < 2) return kFwdEpiWarps;                           // q_full
    if (i >= 3 && i < 7) return 2 + 4 * kFwdGroups;           // ready: two loads, one arrival per softmax warp
    if (i == 20) return kFwdEpiWarps;                         // o_free
    if (i == 21 || i == 22) return 4 * kFwdGroups;            // stats_full
    if (i >= 23 && i < 27) return kFwdGroups;                 // max_full
    return (i >= 11 && i < 15) || i == 19 || (i >= 27 && i < 39) ? 1 : 0;   // sdone, o_full, and the others
  }
};

template <int D> struct WinCta {
  uint8_t *sK, *sV;
  float* smax;
  volatile WinUnitInfo* units;
  uint32_t* redo;
  volatile int* abort_flag;
  uint32_t tmem_base;
};

// What a role knows about unit n once it is listed.  False: no such unit (or a wait has run out).
template <int D>
__device__ __forceinline__ bool win_await_unit(const WinCta<D>& c, const WinBars& bar, int n, WinUnitInfo& u) {
  if (!mbar_wait_spin(bar.listed + n % 4, (n / 4) & 1, c.abort_flag)) return false;
  u.id = c.units[n].id;
  u.tiles = c.units[n].tiles;
  return u.id >= 0;
}

// A listed unit's tiles: it has a query.
__device__ __forceinline__ void win_tiles(const WinFwdArgs& a, const WinUnit& u, int& len, WinTiles& t) {
  len = a.mask.length(u.b);
  t.set(a.mask, u.qt * kTile, len);
}

// ---------------------------------------------------------------------------------- units (a warp)
// Asks the hardware for a CTA that has not been launched yet and takes its place.
__device__ __forceinline__ void queue_ask(void* answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_u32(answer)),
               "r"(smem_u32(bar))
               : "memory");
}
// Its index, or -1 when none was left.
__device__ __forceinline__ int queue_answer(const void* answer) {
  int id;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b128 r;\n"
      "ld.shared.b128 r, [%1];\n"
      "mov.s32 %0, -1;\n"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n"
      "}\n"
      : "=r"(id)
      : "r"(smem_u32(answer))
      : "memory");
  return id;
}

// A unit without a query: zeros and -infinity.
template <int D>
__device__ __forceinline__ void win_clear_unit(const WinFwdArgs& a, const WinUnit& u, int lane) {
  const int rows = min(kTile, a.mask.n - u.qt * kTile);
  const size_t first = static_cast<size_t>(u.b) * a.mask.n + u.qt * kTile;
  for (int i = lane; i < rows * (D / 8); i += 32)
    *reinterpret_cast<uint4*>(a.o + ((first + i / (D / 8)) * a.heads + u.h) * D + i % (D / 8) * 8) = make_uint4(0, 0, 0, 0);
  if (a.lse != nullptr)
    for (int i = lane; i < rows; i += 32)
      a.lse[(static_cast<size_t>(u.b) * a.heads + u.h) * a.mask.n + u.qt * kTile + i] = -INFINITY;
}

// The stream's units: the CTA's own, then what the queue gives; those without a query are dealt with here and never listed.
template <int D>
__device__ __forceinline__ void win_take_units(const WinCta<D>& c, const WinFwdArgs& a, const WinBars& bar, void* answer, int lane) {
  int tiles = 0;   // of the unit listed last
  int asked = 0;
  // the next unit of the queue, -1 if there is none
  auto ask = [&]() {
    if (asked == kWinMaxUnits) return -1;
    int id = -1;
    if (lane == 0) {
      mbar_arrive_expect_tx(bar.answer, 16);
      queue_ask(answer, bar.answer);
    }
    __syncwarp();
    if (mbar_wait_ok(bar.answer, asked & 1, c.abort_flag)) id = queue_answer(answer);
    fence_proxy_async_smem();   // the next answer is written behind this reading
    __syncwarp();
    ++asked;
    return id;
  };
  int id = blockIdx.x, done = 0;   // done: units known to be
  for (int n = 0;; ++n) {
    if (n > 0) {
      // Unit n is asked for when unit n - 2 is done.  Where unit n - 1 is a single tile that would be too late: the last tile of
      // unit n - 2 waits for the K of two tiles on, unit n's.
      bool ok = true;
      for (const int before = tiles == 1 ? n - 2 : n - 1; ok && done < before; ++done)
        ok = mbar_wait_ok(bar.done + done % 4, (done / 4) & 1, c.abort_flag);
      id = ok ? ask() : -1;
    }
    for (; id >= 0; id = ask()) {
      const WinUnit u(a, id);
      if (u.qt * kTile < a.mask.length(u.b)) break;
      win_clear_unit<D>(a, u, lane);
    }
    tiles = 0;
    if (id >= 0) {
      const WinUnit u(a, id);
      WinTiles t;
      t.set(a.mask, u.qt * kTile, a.mask.length(u.b));
      tiles = t.count();
    }
    if (lane == 0) {
      c.units[n].id = id;
      c.units[n].tiles = tiles;
      mbar_arrive(bar.listed + n % 4);
    }
    if (id < 0) break;
  }
}

// ---------------------------------------------------------------------------------- loads
// The CTA's stream of key tiles: per unit the diagonal tile, then the others in ascending order.
template <int D> struct WinStream {
  int n, kt, left;        // unit, its tile at hand, tiles still to come behind that one
  int qt, kvh, b, len;
  bool diagonal;          // the tile at hand is the first, out of order
  WinTiles t;
  __device__ bool open(const WinCta<D>& c, const WinFwdArgs& a, const WinBars& bar) {
    WinUnitInfo u;
    if (!win_await_unit(c, bar, n, u)) return false;
    const WinUnit w(a, u.id);
    win_tiles(a, w, len, t);
    qt = w.qt;
    kvh = a.by_group.quot(w.h);
    b = w.b;
    kt = qt;
    diagonal = true;
    left = u.tiles - 1;
    return true;
  }
  // to the next tile; false behind the last of all
  __device__ bool step(const WinCta<D>& c, const WinFwdArgs& a, const WinBars& bar) {
    if (left == 0) {
      ++n;
      return open(c, a, bar);
    }
    --left;
    kt = diagonal ? t.first() : t.next(kt);
    diagonal = false;
    if (kt == qt) kt = t.next(kt);
    return true;
  }
};

// K of tiles 0 and 1, then K(J+2) as soon as S(J-1) has freed its stage.  One thread.
template <int D>
__device__ __forceinline__ void win_load_k(const WinCta<D>& c, const WinFwdArgs& a, const CUtensorMap* tm, const WinBars& bar) {
  WinStream<D> s;
  s.n = 0;
  bool there = s.open(c, a, bar);
  for (int J = 0, behind = 0; behind < 2; ++J) {   // tile J of the stream; two more arrivals behind the last: the issuer looks ahead
    uint64_t* full = J < 2 ? bar.k_pre + J : bar.ready + (J - 2) % 4;
    if (J >= 3 && !mbar_wait_spin(bar.sdone + (J - 3) % 4, ((J - 3) / 4) & 1, c.abort_flag)) break;
    if (!there) {
      mbar_arrive(full);
      ++behind;
      continue;
    }
    mbar_arrive_expect_tx(full, TileGeom<D>::kBytes);
    tma_load_tile<D>(c.sK + (J % kFwdKStages) * TileGeom<D>::kBytes, tm, full, s.kt * kTile, s.kvh, s.b);
    there = s.step(c, a, bar);
  }
}

// V(J) as soon as S(J-1) is done, and with it P V of tile J-3, which used its stage.  A warp.
template <int D>
__device__ __forceinline__ void win_load_v(const WinCta<D>& c, const WinFwdArgs& a, const CUtensorMap* tm, const WinBars& bar, int lane) {
  WinStream<D> s;
  s.n = 0;
  bool there = __all_sync(0xffffffffu, s.open(c, a, bar));
  int fixes = 0;
  for (int J = 0; there; ++J) {
    if (J >= 3 && !mbar_wait_ok(bar.sdone + (J - 1) % 4, ((J - 1) / 4) & 1, c.abort_flag)) break;
    uint8_t* dst = c.sV + (J % kFwdVStages) * TileGeom<D>::kBytes;
    uint64_t* full = bar.ready + J % 4;
    const int rows = s.len - s.kt * kTile;       // rows of the tile that are keys
    if (rows < kTile && s.len < a.mask.n) {
      if (lane == 0) {
        mbar_arrive_expect_tx(bar.landed, TileGeom<D>::kBytes);
        tma_load_tile<D>(dst, tm, bar.landed, s.kt * kTile, s.kvh, s.b);
      }
      if (!mbar_wait_ok(bar.landed, fixes & 1, c.abort_flag)) break;
      ++fixes;
      zero_rows_by_warp<D>(dst, max(rows, 0), lane);
      if (lane == 0) mbar_arrive(full);
    } else if (lane == 0) {
      mbar_arrive_expect_tx(full, TileGeom<D>::kBytes);
      tma_load_tile<D>(dst, tm, full, s.kt * kTile, s.kvh, s.b);
    }
    there = __all_sync(0xffffffffu, s.step(c, a, bar));
  }
}

// ---------------------------------------------------------------------------------- MMA issuer (one thread)
template <int D>
__device__ __forceinline__ void win_issue(const WinCta<D>& c, const WinBars& bar) {
  const uint64_t k_desc0 = desc_kmajor(smem_u32(c.sK));
  const uint32_t sV_addr = smem_u32(c.sV);
  const uint32_t tmem_base = c.tmem_base;
  volatile int* abort_flag = c.abort_flag;
  constexpr uint32_t idesc_s = make_idesc_bf16(kTile, kTile, false, false), idesc_pv = make_idesc_bf16(kTile, D, false, true);
  uint64_t *ready = bar.ready, *sdone = bar.sdone;
  auto issue_s = [&](int J, int qbuf) {
    const uint32_t qcol = tmem_base + kFwdColQ + qbuf * kFwdQCols;
    const uint64_t k_desc = desc_step(k_desc0, (J % kFwdKStages) * TileGeom<D>::kBytes);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
      mma_ts(tmem_base + kFwdColS + (J % kFwdSBufs) * 128, qcol + k * 8,
             desc_step(k_desc, (k >> 2) * TileGeom<D>::kBlockBytes + (k & 3) * 32), idesc_s, k > 0);
    mma_commit(sdone + J % 4);
  };
  auto issue_pv = [&](int J, bool first) {
    const uint32_t pcol = tmem_base + kFwdColS + (J % kFwdSBufs) * 128;
    const uint64_t v_desc = desc_mnmajor(sV_addr + (J % kFwdVStages) * TileGeom<D>::kBytes, TileGeom<D>::kBlockBytes);
#pragma unroll
    for (int kb = 0; kb < kTile / 16; ++kb) {
      const uint32_t p = pcol + (kb * 16 / kFwdCols) * kFwdCols + (kb * 16 % kFwdCols) / 2;
      mma_ts(tmem_base + kFwdColO, p, desc_step(v_desc, kb * 2048), idesc_pv, (!first || kb > 0) ? 1u : 0u);
    }
  };
  // the next S to issue: tile s_t of unit s_n, which has s_T tiles (0: the unit is not open yet)
  int s_n = 0, s_t = 0, s_T = 0;
  bool more = true, ok = true;
  auto next_s = [&](int J) {          // S(J), if there is such a tile
    if (!more) return;
    if (s_T == 0) {
      WinUnitInfo u;
      if (!win_await_unit(c, bar, s_n, u)) { more = false; return; }
      s_T = u.tiles;
      ok = mbar_wait_spin(bar.q_full + (s_n & 1), (s_n >> 1) & 1, abort_flag) && ok;
      tc_fence_after_sync();
    }
    issue_s(J, s_n & 1);
    if (++s_t == s_T) { s_t = s_T = 0; ++s_n; }
  };
  for (int J = 0; J < 2; ++J) {
    ok = mbar_wait_spin(bar.k_pre + J, 0, abort_flag) && ok;
    tc_fence_after_sync();
    if (ok) next_s(J);
  }
  int J = 0;
  for (int n = 0; ok; ++n) {
    if (!more && n == s_n) break;      // S has met the end: there is no unit n
    const int T = c.units[n].tiles;
    for (int t = 0; t < T && ok; ++t, ++J) {
      if (t > 0 && t + kFwdSBufs < T) {   // inside the unit: nothing to ask about
        do {
          ok = mbar_wait_spin(ready + J % 4, (J / 4) & 1, abort_flag);
          tc_fence_after_sync();
          issue_pv(J, false);
          issue_s(J + kFwdSBufs, n & 1);
          ++t;
          ++J;
        } while (t + kFwdSBufs < T && ok);
        s_n = n + 1;                      // S has issued the unit's last tile
        s_t = s_T = 0;
        if (!ok) break;
      }
      ok = mbar_wait_spin(ready + J % 4, (J / 4) & 1, abort_flag);
      if (t == 0 && n > 0) ok = mbar_wait_spin(bar.o_free, (n - 1) & 1, abort_flag) && ok;   // the previous unit's O is out
      tc_fence_after_sync();
      issue_pv(J, t == 0);
      if (t == T - 1) mma_commit(bar.o_full);
      next_s(J + kFwdSBufs);
    }
  }
}

// ---------------------------------------------------------------------------------- softmax groups
// exp2(s * scale_log2 - m) of a group's 32 keys, those without a bit in `see` 0, as bf16 pairs; returns their sum.
__device__ __forceinline__ float win_exp32(const uint32_t (&s)[32], uint32_t see, float scale_log2, float neg_m, uint32_t (&pk)[16]) {
  const uint64_t sc2 = f32x2(scale_log2, scale_log2), nm2 = f32x2(neg_m, neg_m);
  uint64_t acc_a = f32x2(0.f, 0.f), acc_b = f32x2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < 32; c += 2) {
    float x0, x1;
    f32x2_split(fma2(f32x2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, nm2), x0, x1);
    const float p0 = fast_exp2((see >> c) & 1u ? x0 : -INFINITY), p1 = fast_exp2((see >> (c + 1)) & 1u ? x1 : -INFINITY);
    if ((c >> 1) & 1) acc_a = add2(acc_a, f32x2(p0, p1));
    else acc_b = add2(acc_b, f32x2(p0, p1));
    pk[c >> 1] = pack_bf16(p0, p1);
  }
  float r0, r1;
  f32x2_split(add2(acc_a, acc_b), r0, r1);
  return r0 + r1;
}

// `count` full tiles from tile J of the stream on: the loop in which the kernel spends its time.  Out of line and handed plain
// values, so that its code does not depend on the bookkeeping around it.
__device__ __noinline__ float win_run(uint32_t lane_s, uint32_t sdone, uint32_t ready, uint32_t abort_flag, float scale_log2, float neg_m,
                                      float l_run, int J, int count) {
  static_assert(kFwdCols == 32, "one 32-column load per thread and tile");
  const int lane = threadIdx.x & 31;
  float unused = 0.f;
  for (int i = 0; i < count; ++i, ++J) {
    const uint32_t colS = lane_s + (J % kFwdSBufs) * 128;
    mbar_wait_at(sdone + 8 * (J % 4), (J / 4) & 1, abort_flag);
    tc_fence_after_sync();
    uint32_t sv[32], pk[16];
    tmem_ld32(colS, sv);
    tmem_wait_ld();
    l_run += fwd_exp32(sv, 32, scale_log2, neg_m, pk, unused);
    tmem_st16(colS, pk);   // in place: this thread has read all of its S columns
    tmem_wait_st();
    tc_fence_before_sync();
    warp_arrive_at(ready + 8 * (J % 4), lane);
  }
  return l_run;
}

template <int D>
__device__ __forceinline__ bool win_softmax(const WinCta<D>& c, const WinFwdArgs& a, const WinBars& bar, int warp, int r) {
  const int g = warp >> 2, lane = r & 31;
  const FwdStats<D> stats{c.smax};
  const uint32_t lane_s = c.tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kFwdColS + g * kFwdCols;
  const uint32_t sdone = smem_u32(bar.sdone), ready = smem_u32(bar.ready), abort_at = smem_u32(const_cast<int*>(c.abort_flag));
  bool asked = false;
  int J = 0;
  for (int n = 0;; ++n) {
    WinUnitInfo u;
    if (!__all_sync(0xffffffffu, win_await_unit(c, bar, n, u))) break;
    const WinUnit w(a, u.id);
    int len, lo = 0, hi = 0;
    WinTiles t;
    win_tiles(a, w, len, t);
    const int row = w.qt * kTile + r;
    const bool live = row < len;
    if (live) a.mask.keys_of(row, len, lo, hi);
    const int sink = min(a.mask.sink, hi);
    auto see = [&](int kt) {
      const int base = kt * kTile + g * kFwdCols;
      return bits_below(sink, base) | (bits_below(hi, base) & ~bits_below(lo, base));
    };
    // the diagonal tile comes first and fixes the rows' reference; full tiles in runs, all others, the first too, in one piece of
    // code, since in short calls much of the time goes into fetching instructions
    float m_ref = 0.f, l_run = 0.f;
    bool first = true;
    for (int kt = w.qt; kt < t.w1;) {
      if (!first && kt == w.qt) { kt = t.next(kt); continue; }
      if (!first && t.full(kt)) {
        const int end = t.run_end(kt), count = end - kt - (w.qt >= kt && w.qt < end ? 1 : 0);
        l_run = win_run(lane_s, sdone, ready, abort_at, a.scale_log2, -m_ref, l_run, J, count);
        J += count;
        kt = t.next(end - 1);
        continue;
      }
      const uint32_t colS = lane_s + (J % kFwdSBufs) * 128;
      mbar_wait_at(sdone + 8 * (J % 4), (J / 4) & 1, abort_at);
      tc_fence_after_sync();
      uint32_t s[32], pk[16];
      tmem_ld32(colS, s);
      const uint32_t bits = see(kt);
      tmem_wait_ld();
      // 32 rows by 32 keys of which none is seen: a third of the diagonal tile, most of the sinks'
      const bool any = __any_sync(0xffffffffu, bits != 0u);
      if (first) {
        float mx = -INFINITY;
        if (any) {
#pragma unroll
          for (int k = 0; k < 32; ++k) mx = fmaxf(mx, (bits >> k) & 1u ? __uint_as_float(s[k]) : -INFINITY);
        }
        float* slot = stats.maxima(n);   // alternates: a fast thread may be a unit ahead of the others
        slot[g * kTile + r] = mx;
        warp_arrive(bar.max_full + (warp & 3), lane);
        mbar_wait(bar.max_full + (warp & 3), n & 1, c.abort_flag);
#pragma unroll
        for (int og = 0; og < kFwdGroups; ++og) mx = fmaxf(mx, slot[og * kTile + r]);
        // a live row whose scores are all -infinity or NaN gets an infinite reference, and with it the second pass
        if (live) m_ref = mx * a.scale_log2;
      }
      if (any) {
        l_run += win_exp32(s, bits, a.scale_log2, -m_ref, pk);
      } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) pk[k] = 0u;
      }
      tmem_st16(colS, pk);
      tmem_wait_st();
      tc_fence_before_sync();
      warp_arrive_at(ready + 8 * (J % 4), lane);
      ++J;
      kt = first ? t.first() : t.next(kt);
      first = false;
    }
    // the slots of unit n - 2 are free: the epilogue warps brought Q of unit n after they had read them
    stats.sums(n)[g * kTile + r] = l_run;
    if (g == 0) stats.refs(n)[r] = m_ref;
    if (live && !(l_run < kFastSumLimit)) {   // true for inf and NaN too
      atomicOr(c.redo + (n >> 5), 1u << (n & 31));
      asked = true;
    }
    warp_arrive(bar.stats_full + (n & 1), lane);
  }
  return asked;
}

// ---------------------------------------------------------------------------------- epilogue warps
// 32 accumulator columns of the lane's row times 1/l (or zeros, where the row is not live) as bf16 into its row.
__device__ __forceinline__ void win_store_slice(const uint32_t (&acc)[32], float inv, bool live, uint64_t& chk2, const QuadRows& out,
                                                int col0, int lane) {
  const uint64_t inv2 = f32x2(inv, inv), zero2 = f32x2(0.f, 0.f);
  uint4 ch[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t f2 = mul2(f32x2(__uint_as_float(acc[8 * v + 2 * e]), __uint_as_float(acc[8 * v + 2 * e + 1])), inv2);
      chk2 = fma2(f2, zero2, chk2);
      float f0, f1;
      f32x2_split(f2, f0, f1);
      w[e] = live ? pack_bf16(f0, f1) : 0u;
    }
    ch[v] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  store_quad_rows(ch, out, col0, lane);
}

template <int D>
__device__ __forceinline__ bool win_epilogue(const WinCta<D>& c, const WinFwdArgs& a, const WinBars& bar, int warp, int lane) {
  constexpr int kSlices = D / 32, kOwn = kSlices / 2;
  constexpr int kFirstWarp = 4 * kFwdGroups + 4;
  const FwdStats<D> stats{c.smax};
  const int half = (warp - kFirstWarp) >> 2;
  const int r = (warp & 3) * 32 + lane;
  const uint32_t tmem_lane = c.tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  // Q of unit n.  Every warp arrives, those without a share of Q too: Q of unit n then says that all of them have read the row
  // sums of unit n - 2, whose slots the softmax threads write next.
  auto stage_q = [&](int n) {
    WinUnitInfo u;
    if (!__all_sync(0xffffffffu, win_await_unit(c, bar, n, u))) return false;
    if (D / 64 == 2 || half == 0) {
      const WinUnit w(a, u.id);
      const QuadRows rows = quad_rows_strided(a.q, a.qs, w.b, w.h, a.mask.n, w.qt * kTile + r);
      uint32_t qr[32];
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint4 ch[4];
        load_quad_rows(ch, rows, half * 64 + part * 32, lane);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          qr[16 * part + 4 * v] = ch[v].x; qr[16 * part + 4 * v + 1] = ch[v].y;
          qr[16 * part + 4 * v + 2] = ch[v].z; qr[16 * part + 4 * v + 3] = ch[v].w;
        }
      }
      tmem_st32(tmem_lane + kFwdColQ + (n & 1) * kFwdQCols + half * 32, qr);
      tmem_wait_st();
    }
    tc_fence_before_sync();
    warp_arrive(bar.q_full + (n & 1), lane);
    return true;
  };
  bool asked = false;
  bool there = stage_q(0);
  bool next = there && stage_q(1);
  for (int n = 0; there; ++n) {
    const WinUnit w(a, c.units[n].id);
    const int len = a.mask.length(w.b), row = w.qt * kTile + r;
    const bool live = row < len;
    const QuadRows out = quad_rows(a.o, w.b, w.h, a.mask.n, a.heads, D, row);
    if (!mbar_wait_relaxed_ok(bar.stats_full + (n & 1), (n >> 1) & 1, c.abort_flag)) break;
    float l = 0.f;
#pragma unroll
    for (int g = 0; g < kFwdGroups; ++g) l += stats.sums(n)[g * kTile + r];
    const float m = stats.refs(n)[r], inv = 1.f / l;
    uint64_t chk2 = f32x2(0.f, 0.f);
    if (!mbar_wait_ok(bar.o_full, n & 1, c.abort_flag)) break;
    if (warp == kFirstWarp && lane == 0) mbar_arrive(bar.done + n % 4);
    tc_fence_after_sync();
    uint32_t acc[kOwn][32];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) tmem_ld32(tmem_lane + kFwdColO + (half * kOwn + i) * 32, acc[i]);
    tmem_wait_ld();
    tc_fence_before_sync();
    warp_arrive(bar.o_free, lane);   // the next unit may start on O
#pragma unroll
    for (int i = 0; i < kOwn; ++i) win_store_slice(acc[i], inv, live, chk2, out, (half * kOwn + i) * 32, lane);
    if (half == 0 && row < a.mask.n && a.lse != nullptr)
      a.lse[(static_cast<size_t>(w.b) * a.heads + w.h) * a.mask.n + row] = live ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    if (live && !fwd_all_finite(chk2)) {
      atomicOr(c.redo + (n >> 5), 1u << (n & 31));
      asked = true;
    }
    there = next;
    next = next && stage_q(n + 2);
  }
  return asked;
}

// ---------------------------------------------------------------------------------- second pass
// One unit by the formula, on the ordinary cores: a warp per row, eight lanes per key (D/8 elements each), four keys at a time, running
// maximum.  About 10 ms for a unit of 32000 keys, less where all is NaN.
template <int D>
__device__ __noinline__ void win_careful_unit(const WinFwdArgs& a, int id, int warp, int lane) {
  constexpr int kPer = D / 8;
  const WinUnit u(a, id);
  const int len = a.mask.length(u.b), part = lane & 7, slot = lane >> 3;
  for (int r = warp; r < kTile; r += kWinThreads / 32) {
    const int row = u.qt * kTile + r;
    if (row >= a.mask.n) break;
    __nv_bfloat16* out = a.o + ((static_cast<size_t>(u.b) * a.mask.n + row) * a.heads + u.h) * D;
    float* lse = a.lse == nullptr ? nullptr : a.lse + (static_cast<size_t>(u.b) * a.heads + u.h) * a.mask.n + row;
    float o[kPer], q[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
    if (row < len) {
      const __nv_bfloat16* src = a.q + u.b * a.qs.b + row * a.qs.t + u.h * a.qs.h + part * kPer;
#pragma unroll
      for (int e = 0; e < kPer; ++e) q[e] = __bfloat162float(src[e]);
      int lo, hi;
      a.mask.keys_of(row, len, lo, hi);
      const int sink = min(min(a.mask.sink, hi), lo), keys = sink + hi - lo;   // the sinks in front of the window, then the window
      const __nv_bfloat16* kb = a.k + u.b * a.ks.b + (u.h / a.group) * a.ks.h + part * kPer;
      const __nv_bfloat16* vb = a.v + u.b * a.vs.b + (u.h / a.group) * a.vs.h + part * kPer;
      for (int x = 0; x < keys; x += 4) {
        const bool there = x + slot < keys;
        const int y = there ? x + slot : keys - 1, j = y < sink ? y : lo + y - sink;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) s = fmaf(q[e], __bfloat162float(kb[j * a.ks.t + e]), s);
#pragma unroll
        for (int d = 1; d < 8; d *= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= a.scale_log2;
        // a NaN score makes everything NaN: nothing to add to that
        if ((x & 127) == 0 && __any_sync(0xffffffffu, isnan(l))) break;
        if (there) {
          const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
          const float alpha = fast_exp2(m - ref), p = fast_exp2(s - ref);
          m = top;
          l = l * alpha + p;
#pragma unroll
          for (int e = 0; e < kPer; ++e) o[e] = fmaf(p, __bfloat162float(vb[j * a.vs.t + e]), o[e] * alpha);
        }
      }
#pragma unroll
      for (int d = 8; d < 32; d *= 2) {   // the four slots of the warp
        const float m2 = __shfl_xor_sync(0xffffffffu, m, d), l2 = __shfl_xor_sync(0xffffffffu, l, d);
        const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
        const float w1 = fast_exp2(m - ref), w2 = fast_exp2(m2 - ref);
        l = l * w1 + l2 * w2;
        m = top;
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = o[e] * w1 + __shfl_xor_sync(0xffffffffu, o[e], d) * w2;
      }
    }
    const float inv = row < len ? 1.f / l : 0.f;
    if (slot == 0) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) out[part * kPer + e] = __float2bfloat16_rn(row < len ? o[e] * inv : 0.f);
      if (part == 0 && lse != nullptr) *lse = row < len ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
  }
}

// ---------------------------------------------------------------------------------- kernel
template <int D>
__global__ void __launch_bounds__(kWinThreads, 1)
window_attn_fwd_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const __grid_constant__ WinFwdArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align_1024(smem_raw);
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(smem + WinFwdSmem<D>::kBars);
  const WinBars bar(bar_mem);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(smem + WinFwdSmem<D>::kHolder);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t kTmemCols = 512;
  constexpr int kMmaWarp = 4 * kFwdGroups, kUnitWarp = kMmaWarp + 1, kKWarp = kMmaWarp + 2, kVWarp = kMmaWarp + 3;

  if (a.careful) {
    win_careful_unit<D>(a, blockIdx.x, warp, lane);
    return;
  }
  WinCta<D> c;
  c.sK = smem + WinFwdSmem<D>::kK;
  c.sV = smem + WinFwdSmem<D>::kV;
  c.smax = reinterpret_cast<float*>(smem + WinFwdSmem<D>::kMax);
  c.units = reinterpret_cast<volatile WinUnitInfo*>(smem + WinFwdSmem<D>::kUnits);
  c.redo = reinterpret_cast<uint32_t*>(smem + WinFwdSmem<D>::kRedo);
  c.abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  if (warp == kKWarp && lane == 0) { tma_prefetch_desc(&tm_k); tma_prefetch_desc(&tm_v); }
  if (tid < kWinBarSlots) {
    const int arrivals = WinBars::arrivals(tid);
    if (arrivals > 0) mbar_init(bar_mem + tid, arrivals);
    fence_mbar_init();
  }
  if (tid == 0) *c.abort_flag = 0;
  if (tid <= kWinMaxUnits / 32) c.redo[tid] = 0;
  fence_proxy_async_smem();
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  c.tmem_base = *tmem_holder;

  bool asked = false;
  if (warp < kMmaWarp) asked = win_softmax<D>(c, a, bar, warp, tid & 127);
  else if (warp == kMmaWarp) { if (lane == 0) win_issue<D>(c, bar); }
  else if (warp == kUnitWarp) win_take_units<D>(c, a, bar, smem + WinFwdSmem<D>::kAnswer, lane);
  else if (warp == kKWarp) { if (lane == 0) win_load_k<D>(c, a, &tm_k, bar); }
  else if (warp == kVWarp) win_load_v<D>(c, a, &tm_v, bar, lane);
  else asked = win_epilogue<D>(c, a, bar, warp, lane);
  __syncwarp();
  // every MMA has finished by now: the epilogue warps waited for the last one
  tc_fence_before_sync();
  if (__syncthreads_or(asked) && !*c.abort_flag) {
    for (int n = 0; c.units[n].id >= 0; ++n)
      if ((c.redo[n >> 5] >> (n & 31)) & 1u) win_careful_unit<D>(a, c.units[n].id, warp, lane);
  }
  settle_after_abort(c.abort_flag);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(c.tmem_base, kTmemCols);
}

}  // namespace astro
