// Forward of attention over lists of key blocks: O and LSE.
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - LSE_i),  j over the tokens of the blocks listed for i's query block
//
// The work of a listed block is that of a block of dense attention, so the kernel is built like the dense forward: one
// CTA per SM walks over its share of the units (a 128-query tile of one head of one sample), the key tiles of all its
// units form one stream, four softmax groups of 128 threads, one thread that issues every tcgen05 MMA, one
// warp that follows the lists, a thread each for the loads of K and V, eight warps that bring Q and take O out.  What the dense
// kernel knows beforehand (how many tiles a unit has, which keys of a tile exist) is here data: the producer warp writes a
// descriptor per tile, a few tiles ahead, and the other roles act on it.  Tensor-memory layout, the S look-ahead, the rings and
// the one-wait, one-commit rhythm of the issuing thread are the dense kernel's.
//
// Precision: bf16 products, fp32 sums.  P is rounded to bf16 for P V (half a step, 2^-8 of each weight at most), the row sum is taken from the
// fp32 values.  Fast pass: each row keeps the maximum of its unit's first tile as its one reference; exp2(s - m) is exact for
// any reference as long as nothing overflows.  A unit with a row sum beyond 2^100, an infinity or a NaN, or whose first tile gives
// a row no finite score, is done again by the careful pass: a plain loop, tile by tile, with the running maximum of the textbook.
//
// Bound: the tensor pipe and its hand-offs.  A tile takes 1600 to 1670 clocks (the dense kernel's 1630), of which the MMAs are
// 1024: S -> softmax 1250 -> hand-over 300 -> P V and the next S 1250, two tiles in flight.  Layer shape, 64 of 273 blocks of
// 120 tokens per query block: 203 to 210 us in short bursts = 1050 to 1090 TFLOP/s (tensor pipe 58 %, DRAM bytes as few as the inputs
// and outputs have), 242 us in a loop under the power limit (993 W, 1.53 GHz, 370k clocks).  With every query block naming one and the
// same block 205 us, and 218 us in the loop (992 W, 1.66 GHz, 362k clocks): random lists cost 2 % in clocks and, where power is
// the limit, 8 % in clock rate.  Start and end of the kernel take 9 % of its clocks, a unit boundary 2.5 tiles.
// Registers: 72 per thread (27 warps); the softmax loop spills nothing, the other roles' code 212 bytes, 11 local accesses per key tile of
// 3600 warp instructions.
//
// Few units: a unit's list is cut into up to `splits` ranges that run as units of their own and leave O (fp32, normalised)
// and LSE of their part; sparse_combine_kernel joins them.
#pragma once
#include "attn_fwd.cuh"
#include "sparse_common.cuh"

namespace astro {

struct SparseUnits {
  int q_tiles, dim_y, cache_shared, splits, entries, n_select;   // entries: list entries per split
  int first, stride, total;
};
// Unit id -> (query tile, head, sample, split); query tiles fastest, then (y, z) = (head, sample), or (sample, head) when one
// stored prefix serves every sample (see the dense kernel), splits slowest.
struct SparseUnit {
  int qt, h, b, split;
  __device__ SparseUnit(const SparseUnits& s, int unit, int heads, int batch) {
    qt = unit % s.q_tiles;
    int x = unit / s.q_tiles;
    const int y = x % s.dim_y;
    x /= s.dim_y;
    const int dim_z = s.cache_shared ? heads : batch;
    const int z = x % dim_z;
    split = x / dim_z;
    h = s.cache_shared ? z : y;
    b = s.cache_shared ? y : z;
  }
};

struct SparseFwdArgs {
  const __nv_bfloat16* q;
  const int* blocks;       // [B][H][q_tiles][n_select]
  __nv_bfloat16* o;
  float* lse;              // may be null
  float* part_o;           // [split][B][H][n_q][D] when splits > 1
  float* part_lse;         // [split][B][H][n_q]
  int batch, heads, n_q;
  float scale_log2;
  int careful;             // 1: careful pass only
};

template <int D> struct SparseFwdSmem {
  static constexpr int kK = FwdSmem<D>::kK;
  static constexpr int kV = FwdSmem<D>::kV;
  static constexpr int kMax = FwdSmem<D>::kMax;
  static constexpr int kBars = FwdSmem<D>::kBars;                            // 48 barriers, holder and abort flag
  static constexpr int kDesc = kBars + 48 * 8 + 16;
  static constexpr int kSource = kDesc + kSpDescs * static_cast<int>(sizeof(TileDesc));
  static constexpr int kRedo = kSource + kSpDescs * static_cast<int>(sizeof(TileSource));
  static constexpr int kTotal = kRedo + kFwdMaxUnits / 8 + 1024;
};

// Everything a role needs.
template <int D> struct SparseCta {
  uint8_t *sK, *sV;
  float* smax;
  TileDesc* desc;
  TileSource* source;
  uint32_t* redo;
  volatile int* abort_flag;
  uint32_t tmem_base;
};

// The units of a CTA as one stream of tiles (list warp, all lanes).  The first entries of the next unit's list are
// asked for when a unit is opened.
struct SparseStream {
  ListWalker w;
  const int* list;        // of the unit to open next
  int unit, count, first; // its id, length and first entries
  int h, b, bx;           // of the open unit
  uint32_t live;
  bool opens;
  // `unit` is the one to open next: where its list is, and its first entries
  __device__ void look_up(const SparseUnits& s, const SparseFwdArgs& a, int lane) {
    if (unit >= s.total) return;
    const SparseUnit u(s, unit, a.heads, a.batch);
    const int from = u.split * s.entries;
    list = a.blocks + ((static_cast<long long>(u.b) * a.heads + u.h) * s.q_tiles + u.qt) * s.n_select + from;
    count = max(0, min(s.entries, s.n_select - from));
    first = ListWalker::first_entries(list, count, lane);
  }
  __device__ void start(const SparseUnits& s, const SparseFwdArgs& a, int unit_, int lane) {
    unit = unit_;
    look_up(s, a, lane);
  }
  __device__ void open(const SparseGeom& g, const SparseUnits& s, const SparseFwdArgs& a, int lane) {
    const SparseUnit u(s, unit, a.heads, a.batch);
    h = u.h;
    b = u.b;
    bx = s.cache_shared ? 0 : u.b;
    live = live_quarters(a.n_q, u.qt) << kTileLiveShift;
    w.open(g, list, count, lane, first);
    opens = true;
    unit += s.stride;
    look_up(s, a, lane);
  }
};

// The dense fast pass's barriers, one per descriptor (written), and one per warp quarter for the first tile's row maxima:
// every meeting of the fast pass is an mbarrier with a bounded wait, so a role that gives up leaves none of the others
// behind.  ready[J % 4] takes two arrivals with byte counts, V(J)'s and K(J+2)'s.
struct SparseBars : FwdFastBars {
  uint64_t *max_full, *listed;   // [4], kFwdGroups arrivals; [kSpDescs]
  __device__ explicit SparseBars(uint64_t* b) : FwdFastBars(b), max_full(b + 23), listed(b + 27) {}
  // Arrivals of the barrier in slot i (0: none there); every barrier is set up by a thread of its own.
  static __device__ int arrivals(int i) {
    if (i < 2) return kFwdEpiWarps;                           // q_full
    if (i == 2) return 2;                                     // k01: two loads
    if (i >= 3 && i < 7) return 2 + 4 * kFwdGroups;           // ready: two loads, one arrival per softmax warp
    if (i == 20) return kFwdEpiWarps;                         // o_free
    if (i == 21 || i == 22) return 4 * kFwdGroups;            // stats_full
    if (i >= 23 && i < 27) return kFwdGroups;                 // max_full
    return (i >= 11 && i < 15) || i == 19 || (i >= 27 && i < 27 + kSpDescs) ? 1 : 0;   // sdone, o_full, listed
  }
};
constexpr int kSparseBarSlots = 36;
constexpr int kSparseThreads = kFwdThreads + 64;   // the dense kernel's warps and two for the loads of K and V

// O (+)= P V: P of 16 keys = 8 packed columns; group g's pairs start at its own S columns.  One thread.
template <int D>
__device__ __forceinline__ void sparse_pv(uint32_t tmem_base, uint32_t pcol, uint32_t v_smem, uint32_t onto) {
  constexpr uint32_t idesc = make_idesc_bf16(kTile, D, false, true);
  const uint64_t v_desc = desc_mnmajor(v_smem, TileGeom<D>::kBlockBytes);
#pragma unroll
  for (int kb = 0; kb < kTile / 16; ++kb) {
    const uint32_t p = pcol + (kb * 16 / kFwdCols) * kFwdCols + (kb * 16 % kFwdCols) / 2;
    mma_ts(tmem_base + kFwdColO, p, desc_step(v_desc, kb * 2048), idesc, kb > 0 ? 1u : onto);
  }
}
// S = Q K^T of one tile into the S buffer at column `scol`.  One thread.
template <int D>
__device__ __forceinline__ void sparse_s(uint32_t scol, uint32_t qcol, uint64_t k_desc) {
  constexpr uint32_t idesc = make_idesc_bf16(kTile, kTile, false, false);
#pragma unroll
  for (int k = 0; k < D / 16; ++k)   // 16 elements of the head dimension = 8 packed Q columns
    mma_ts(scol, qcol + k * 8, desc_step(k_desc, (k >> 2) * TileGeom<D>::kBlockBytes + (k & 3) * 32), idesc, k > 0);
}

// ---------------------------------------------------------------------------------- producers, fast pass
// Three warps: one follows the lists and writes descriptors and sources, up to four tiles ahead of S; one thread loads K, one
// V.  A single producer needed about 1700 clocks per tile for both jobs, with the loads behind each other in front of an
// MMA that takes 1024 (a 7680-key list per query block, layer shape: 244 us against 217 with the three).

// The list walker.  Tile J overwrites what was written for tile J-8; S(J-4) done means that every P(J-6) has arrived.
// (The wait names the barrier that S(J) will use next, so its phase cannot run ahead of it.)
template <int D>
__device__ __forceinline__ void sparse_walk(const SparseCta<D>& c, const SparseGeom& g, const SparseUnits& s, const SparseFwdArgs& a,
                                            const SparseBars& bar, SparseStream& st, int lane) {
  int J = 0;
  bool over = false;
  // a slot of the rings; false once a wait has run out
  auto slot = [&]() { return J < 4 || mbar_wait_ok(bar.sdone + J % 4, ((J - 4) / 4) & 1, c.abort_flag); };
  while (!over) {
    st.open(g, s, a, lane);
    const bool last_unit = st.unit >= s.total;
    for (bool last = false; !last; ++J) {
      if (!slot()) return;
      uint32_t valid;
      last = next_tile(g, st.w, st.h, st.b, st.bx, c.source + J % kSpDescs, valid);
      if (lane == 0) {
        c.desc[J % kSpDescs].valid = valid;
        c.desc[J % kSpDescs].flags = kTileThere | (st.opens ? kTileFirst : 0u) | (last ? kTileLast : 0u) |
                                     (last && last_unit ? kTileEnd : 0u) | st.live;
        mbar_arrive(bar.listed + J % kSpDescs);
      }
      st.opens = false;
    }
    over = last_unit;
  }
  for (int behind = 0; behind < 2; ++behind, ++J) {   // behind the last tile: the issuer looks two ahead
    if (!slot()) return;
    if (lane == 0) {
      c.desc[J % kSpDescs].flags = 0;
      mbar_arrive(bar.listed + J % kSpDescs);
    }
  }
}

// K of tiles 0 and 1, then K(J+2) as soon as S(J-1) has freed its stage.  One thread.
template <int D>
__device__ __forceinline__ void sparse_load_k(const SparseCta<D>& c, const SparseGeom& g, const SparseMaps& maps,
                                              const SparseBars& bar) {
  const uint32_t bytes = sparse_tile_bytes<D>(g);
  const volatile TileDesc* desc = c.desc;
  auto listed = [&](int J) { return mbar_wait_spin(bar.listed + J % kSpDescs, (J / kSpDescs) & 1, c.abort_flag); };
  auto load = [&](int J, uint64_t* full) {
    load_sparse_tile<D>(c.sK + (J % kFwdKStages) * TileGeom<D>::kBytes, &maps.kx, &maps.kc, full, c.source + J % kSpDescs, g);
  };
  if (!listed(0)) return;
  uint32_t now = desc[0].flags, next = 0;
  mbar_arrive_expect_tx(bar.k01, bytes);
  load(0, bar.k01);
  if (!listed(1)) return;
  next = desc[1].flags;
  if (next & kTileThere) {
    mbar_arrive_expect_tx(bar.k01, bytes);
    load(1, bar.k01);
  } else {
    mbar_arrive(bar.k01);
  }
  for (int J = 0; now & kTileThere; ++J) {
    if (!listed(J + 2)) break;
    const uint32_t later = desc[(J + 2) % kSpDescs].flags;
    uint64_t* full = bar.ready + J % 4;
    if (later & kTileThere) {
      if (J >= 1 && !mbar_wait_spin(bar.sdone + (J - 1) % 4, ((J - 1) / 4) & 1, c.abort_flag)) break;
      mbar_arrive_expect_tx(full, bytes);
      load(J + 2, full);
    } else {
      mbar_arrive(full);
    }
    now = next;
    next = later;
  }
}

// V(J) as soon as S(J-1) is done, and with it P V of tile J-3, which used its stage.  One thread.
template <int D>
__device__ __forceinline__ void sparse_load_v(const SparseCta<D>& c, const SparseGeom& g, const SparseMaps& maps,
                                              const SparseBars& bar) {
  const uint32_t bytes = sparse_tile_bytes<D>(g);
  const volatile TileDesc* desc = c.desc;
  for (int J = 0;; ++J) {
    if (!mbar_wait_spin(bar.listed + J % kSpDescs, (J / kSpDescs) & 1, c.abort_flag)) break;
    const uint32_t flags = desc[J % kSpDescs].flags;
    if (J >= 3 && !mbar_wait_spin(bar.sdone + (J - 1) % 4, ((J - 1) / 4) & 1, c.abort_flag)) break;
    uint64_t* full = bar.ready + J % 4;
    mbar_arrive_expect_tx(full, bytes);
    load_sparse_tile<D>(c.sV + (J % kFwdVStages) * TileGeom<D>::kBytes, &maps.vx, &maps.vc, full, c.source + J % kSpDescs, g);
    if (flags & kTileEnd) break;
  }
}

// ---------------------------------------------------------------------------------- MMA issuer, fast pass (one thread)
template <int D>
__device__ __forceinline__ void sparse_issue(const SparseCta<D>& c, const SparseBars& bar) {
  const uint64_t k_desc0 = desc_kmajor(smem_u32(c.sK));
  const uint32_t sV_addr = smem_u32(c.sV);
  const uint32_t tmem_base = c.tmem_base;
  volatile int* abort_flag = c.abort_flag;
  uint64_t *q_full = bar.q_full, *ready = bar.ready, *sdone = bar.sdone, *o_full = bar.o_full, *o_free = bar.o_free;
  const volatile TileDesc* desc = c.desc;
  auto issue_s = [&](int J, int qbuf) {
    sparse_s<D>(tmem_base + kFwdColS + (J % kFwdSBufs) * 128, tmem_base + kFwdColQ + qbuf * kFwdQCols,
                desc_step(k_desc0, (J % kFwdKStages) * TileGeom<D>::kBytes));
    mma_commit(sdone + J % 4);
  };
  int s_n = 0;   // unit (counted within the CTA) of the last S issued
  auto wait_q = [&]() {
    mbar_wait_spin(q_full + (s_n & 1), (s_n >> 1) & 1, abort_flag);
    tc_fence_after_sync();
  };
  mbar_wait_spin(bar.k01, 0, abort_flag);
  uint32_t now = desc[0].flags, next = desc[1].flags;
  wait_q();
  issue_s(0, 0);
  if (next & kTileThere) {
    if (next & kTileFirst) { ++s_n; wait_q(); }
    issue_s(1, s_n & 1);
  }
  int n = 0;
  for (int J = 0;; ++J) {
    if (!mbar_wait_spin(ready + J % 4, (J / 4) & 1, abort_flag)) break;
    if ((now & kTileFirst) && n > 0) mbar_wait_spin(o_free, (n - 1) & 1, abort_flag);   // the previous unit's O is out
    tc_fence_after_sync();
    const uint32_t later = desc[(J + 2) % kSpDescs].flags;   // its writing was awaited by the K loader's arrival for tile J
    sparse_pv<D>(tmem_base, tmem_base + kFwdColS + (J % kFwdSBufs) * 128, sV_addr + (J % kFwdVStages) * TileGeom<D>::kBytes,
                 (now & kTileFirst) ? 0u : 1u);
    if (now & kTileLast) { mma_commit(o_full); ++n; }
    if (later & kTileThere) {
      if (later & kTileFirst) { ++s_n; wait_q(); }
      issue_s(J + 2, s_n & 1);
    }
    if (now & kTileEnd) break;
    now = next;
    next = later;
  }
}

// ---------------------------------------------------------------------------------- softmax groups, fast pass
// exp2(s * scale_log2 - m) of a group's 32 keys of which the first `valid` exist (the others get 0), as bf16 pairs; returns
// their sum.  The short case selects arguments and leaves the rest of the code as it is in the full one: with a branch per
// eight keys it took 1670 clocks from S to P against 1250, and set the pace of blocks of 120 tokens.
__device__ __forceinline__ float sparse_exp32(const uint32_t (&s)[32], int valid, float scale_log2, float neg_m,
                                              uint32_t (&pk)[16]) {
  float unused = 0.f;
  if (valid >= 32) return fwd_exp32(s, 32, scale_log2, neg_m, pk, unused);
  const uint64_t sc2 = f32x2(scale_log2, scale_log2), nm2 = f32x2(neg_m, neg_m);
  uint64_t acc_a = f32x2(0.f, 0.f), acc_b = f32x2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < 32; c += 2) {
    float x0, x1;
    f32x2_split(fma2(f32x2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, nm2), x0, x1);
    const float p0 = fast_exp2(c < valid ? x0 : -INFINITY), p1 = fast_exp2(c + 1 < valid ? x1 : -INFINITY);
    if ((c >> 1) & 1) acc_a = add2(acc_a, f32x2(p0, p1));
    else acc_b = add2(acc_b, f32x2(p0, p1));
    pk[c >> 1] = pack_bf16(p0, p1);
  }
  float r0, r1;
  f32x2_split(add2(acc_a, acc_b), r0, r1);
  return r0 + r1;
}

__device__ __forceinline__ float row_max(const uint32_t (&s)[32], int valid) {
  float mx = -INFINITY;
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if (k < valid) mx = fmaxf(mx, __uint_as_float(s[k]));
  return mx;
}

// Shared-memory addresses (32 bits) that the softmax loop works with, for one group.
struct SparseLoop {
  uint32_t lane_s, sdone, ready, listed, desc, abort_flag;
  int g;
};
__device__ __forceinline__ TileDesc load_desc(uint32_t desc, int J) {
  TileDesc d;
  asm volatile("ld.volatile.shared::cta.v2.u32 {%0, %1}, [%2];"
               : "=r"(d.valid), "=r"(d.flags)
               : "r"(desc + (J % kSpDescs) * static_cast<uint32_t>(sizeof(TileDesc)))
               : "memory");
  return d;
}
__device__ __forceinline__ TileDesc await_desc(const SparseLoop& c, int J) {
  mbar_wait_at(c.listed + 8 * (J % kSpDescs), (J / kSpDescs) & 1, c.abort_flag);
  return load_desc(c.desc, J);
}

struct SparseRun {
  float l_run;
  int J;
  TileDesc d;   // of tile J
  bool ok;
};
// The tiles of a unit behind its first, from tile J (descriptor d) to the unit's last: the loop in which the kernel spends
// its time.  Out of line and handed plain values, so that its code does not depend on the bookkeeping around it.
__device__ __noinline__ SparseRun sparse_run(SparseLoop c, float scale_log2, float neg_m, float l_run, int J, TileDesc d) {
  static_assert(kFwdCols == 32, "one 32-column load per thread and tile");
  const int lane = threadIdx.x & 31;
  bool ok = true;
  while (true) {
    const uint32_t colS = c.lane_s + (J % kFwdSBufs) * 128;
    const int valid = (d.valid >> (8 * c.g)) & 0xff;
    ok = mbar_wait_at_ok(c.sdone + 8 * (J % 4), (J / 4) & 1, c.abort_flag);
    tc_fence_after_sync();
    uint32_t sv[32], pk[16];
    tmem_ld32(colS, sv);
    const TileDesc next = d.flags & kTileLast ? d : await_desc(c, J + 1);   // long written; in the shadow of the load
    tmem_wait_ld();
    l_run += sparse_exp32(sv, valid, scale_log2, neg_m, pk);
    tmem_st16(colS, pk);   // in place: this thread has read all of its S columns
    tmem_wait_st();
    tc_fence_before_sync();
    warp_arrive_at(c.ready + 8 * (J % 4), lane);
    if ((d.flags & kTileLast) || !ok) break;
    d = next;
    ++J;
  }
  return SparseRun{l_run, J, d, ok};
}

// The whole of a unit for a warp whose quarter of the query tile holds no query: it keeps the hand-offs going and leaves S
// where P would be.  Rows of an MMA do not mix, so what comes of it stays in rows that nobody stores.
__device__ __noinline__ SparseRun sparse_idle(SparseLoop c, int J, TileDesc d) {
  const int lane = threadIdx.x & 31;
  bool ok = true;
  while (true) {
    ok = mbar_wait_at_ok(c.sdone + 8 * (J % 4), (J / 4) & 1, c.abort_flag);
    warp_arrive_at(c.ready + 8 * (J % 4), lane);
    if ((d.flags & kTileLast) || !ok) break;
    ++J;
    d = await_desc(c, J);
  }
  return SparseRun{1.f, J, d, ok};
}

// Returns whether this thread asked for a unit to be done again.
template <int D>
__device__ __forceinline__ bool sparse_softmax(const SparseCta<D>& c, const SparseBars& bar, int warp, int r, float scale_log2) {
  const int g = warp >> 2, lane = r & 31;
  const FwdStats<D> stats{c.smax};
  volatile int* abort_flag = c.abort_flag;
  SparseLoop lp;
  lp.lane_s = c.tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kFwdColS + g * kFwdCols;
  lp.sdone = smem_u32(bar.sdone); lp.ready = smem_u32(bar.ready); lp.listed = smem_u32(bar.listed);
  lp.desc = smem_u32(c.desc);
  lp.abort_flag = smem_u32(const_cast<int*>(abort_flag));
  lp.g = g;
  TileDesc d = await_desc(lp, 0);
  int J = 0;
  bool asked = false;
  int maxima = 0;   // units for which this warp has met the other groups over the row maxima
  for (int n = 0;; ++n) {
    float m_ref = 0.f, l_run;
    uint32_t flags = d.flags;
    bool ok;
    TileDesc next;
    if ((flags >> kTileLiveShift & 7u) <= static_cast<uint32_t>(warp & 3)) {
      const SparseRun run = sparse_idle(lp, J, d);
      l_run = run.l_run;
      J = run.J;
      flags = run.d.flags;
      ok = run.ok;
      next = await_desc(lp, J + 1);
    } else {
    // the unit's first tile fixes the rows' reference
    const int valid = (d.valid >> (8 * g)) & 0xff;
    const uint32_t colS = lp.lane_s + (J % kFwdSBufs) * 128;
    ok = mbar_wait_at_ok(lp.sdone + 8 * (J % 4), (J / 4) & 1, lp.abort_flag);
    tc_fence_after_sync();
    uint32_t s[32], pk[16];
    tmem_ld32(colS, s);
    tmem_wait_ld();
    float* slot = stats.maxima(n);   // alternates: a fast thread may be a unit ahead of the others
    float mx = row_max(s, valid);
    slot[g * kTile + r] = mx;
    warp_arrive(bar.max_full + (warp & 3), lane);
    ok = mbar_wait_ok(bar.max_full + (warp & 3), maxima & 1, abort_flag) && ok;
    ++maxima;
#pragma unroll
    for (int og = 0; og < kFwdGroups; ++og) mx = fmaxf(mx, slot[og * kTile + r]);
    // 0 for the empty list's tile alone.  Keys whose scores are all -infinity leave -infinity, and with it an infinite or NaN row
    // sum: 0 would be no reference for the tiles to come, whose scores may lie far below it.
    m_ref = d.valid == 0u ? 0.f : mx * scale_log2;
    l_run = sparse_exp32(s, valid, scale_log2, -m_ref, pk);
    tmem_st16(colS, pk);
    tmem_wait_st();
    tc_fence_before_sync();
    warp_arrive_at(lp.ready + 8 * (J % 4), lane);
    next = await_desc(lp, J + 1);
    if (ok && !(flags & kTileLast)) {
      const SparseRun run = sparse_run(lp, scale_log2, -m_ref, l_run, J + 1, next);
      l_run = run.l_run;
      J = run.J;
      flags = run.d.flags;
      ok = run.ok;
      next = await_desc(lp, J + 1);
    }
    }
    // the slots of unit n - 2 are free: the epilogue warps brought Q of unit n after they had read them
    stats.sums(n)[g * kTile + r] = l_run;
    if (g == 0) stats.refs(n)[r] = m_ref;
    if (!(l_run < kFastSumLimit)) {   // true for inf and NaN too
      atomicOr(c.redo + (n >> 5), 1u << (n & 31));
      asked = true;
    }
    warp_arrive(bar.stats_full + (n & 1), lane);
    if ((flags & kTileEnd) || !ok) break;
    d = next;
    ++J;
  }
  return asked;
}

// ---------------------------------------------------------------------------------- results of a unit
// Where a lane's row goes: bf16 rows of O (its quad's rows together) and LSE, or the fp32 parts of a split.
template <int D> struct SparseRow {
  bool in_range;
  float *lse_dst, *part;
  QuadRows out, q_rows;
  __device__ SparseRow(const SparseUnits& s, const SparseUnit& u, const SparseFwdArgs& a, int r) {
    const int row = u.qt * kTile + r;
    in_range = row < a.n_q;
    const size_t at = (static_cast<size_t>(u.b) * a.heads + u.h) * a.n_q + (in_range ? row : 0);
    const size_t rows = static_cast<size_t>(a.batch) * a.heads * a.n_q;
    lse_dst = s.splits > 1 ? a.part_lse + u.split * rows + at : a.lse ? a.lse + at : nullptr;
    part = s.splits > 1 ? a.part_o + (u.split * rows + at) * D : nullptr;
    out = quad_rows(a.o, u.b, u.h, a.n_q, a.heads, D, row);
    q_rows = quad_rows(a.q, u.b, u.h, a.n_q, a.heads, D, row);
  }
  // 32 accumulator columns from col0 on, times 1 / l
  __device__ void store(const uint32_t (&acc)[32], float inv, uint64_t& chk2, int col0, int lane) const {
    if (part == nullptr) {
      fwd_store_slice(acc, f32x2(inv, inv), chk2, out, col0, lane);
      return;
    }
    float4* dst = reinterpret_cast<float4*>(part + col0);
#pragma unroll
    for (int c = 0; c < 32; c += 4) {
      const float4 v = make_float4(__uint_as_float(acc[c]) * inv, __uint_as_float(acc[c + 1]) * inv,
                                   __uint_as_float(acc[c + 2]) * inv, __uint_as_float(acc[c + 3]) * inv);
      chk2 = fma2(f32x2(v.x, v.y), f32x2(0.f, 0.f), chk2);
      chk2 = fma2(f32x2(v.z, v.w), f32x2(0.f, 0.f), chk2);
      if (in_range) dst[c / 4] = v;
    }
  }
  __device__ void store_lse(float m, float l) const {
    if (in_range && lse_dst != nullptr) *lse_dst = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
  __device__ void stage_q(uint32_t tmem_q, int part64, int lane) const {
    uint32_t qr[32];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint4 ch[4];
      load_quad_rows(ch, q_rows, part64 * 64 + half * 32, lane);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        qr[16 * half + 4 * v] = ch[v].x; qr[16 * half + 4 * v + 1] = ch[v].y;
        qr[16 * half + 4 * v + 2] = ch[v].z; qr[16 * half + 4 * v + 3] = ch[v].w;
      }
    }
    tmem_st32(tmem_q + part64 * 32, qr);
    tmem_wait_st();
  }
};

template <int D>
__device__ __forceinline__ bool sparse_epilogue(const SparseCta<D>& c, const SparseUnits& s, const SparseFwdArgs& a,
                                                const SparseBars& bar, int warp, int lane) {
  constexpr int kSlices = D / 32, kOwn = kSlices / 2;
  constexpr int kMmaWarp = 4 * kFwdGroups;
  const FwdStats<D> stats{c.smax};
  const int half = (warp - kMmaWarp - 2) >> 2;
  const int r = (warp & 3) * 32 + lane;
  const uint32_t tmem_lane = c.tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  // Every warp arrives, those without a share of Q too: Q of unit n then says that all of them have read the row sums of unit
  // n - 2, whose slots the softmax threads write next.
  auto stage_q = [&](int unit, int buf) {
    if (unit >= s.total) return;
    if (D / 64 == 2 || half == 0)
      SparseRow<D>(s, SparseUnit(s, unit, a.heads, a.batch), a, r).stage_q(tmem_lane + kFwdColQ + buf * kFwdQCols, half, lane);
    tc_fence_before_sync();
    warp_arrive(bar.q_full + buf, lane);
  };
  stage_q(s.first, 0);
  if (s.total - s.first > s.stride) stage_q(s.first + s.stride, 1);
  bool asked = false;
  int n = 0;
  for (int unit = s.first; unit < s.total; unit += s.stride, ++n) {
    const SparseRow<D> row(s, SparseUnit(s, unit, a.heads, a.batch), a, r);
    if (!mbar_wait_relaxed_ok(bar.stats_full + (n & 1), (n >> 1) & 1, c.abort_flag)) break;
    float l = 0.f;
#pragma unroll
    for (int g = 0; g < kFwdGroups; ++g) l += stats.sums(n)[g * kTile + r];
    const float m = stats.refs(n)[r];
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint64_t chk2 = f32x2(0.f, 0.f);
    if (!mbar_wait_ok(bar.o_full, n & 1, c.abort_flag)) break;
    tc_fence_after_sync();
    uint32_t acc[kOwn][32];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) tmem_ld32(tmem_lane + kFwdColO + (half * kOwn + i) * 32, acc[i]);
    tmem_wait_ld();
    tc_fence_before_sync();
    warp_arrive(bar.o_free, lane);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) row.store(acc[i], inv, chk2, (half * kOwn + i) * 32, lane);
    if (half == 0) row.store_lse(m, l);
    if (row.in_range && !fwd_all_finite(chk2)) {
      atomicOr(c.redo + (n >> 5), 1u << (n & 31));
      asked = true;
    }
    if (s.total - unit > 2 * s.stride) stage_q(unit + 2 * s.stride, n & 1);
  }
  return asked;
}

// ---------------------------------------------------------------------------------- careful pass
// One unit, tile by tile, nothing overlapped: load, S, running maximum, P, P V.  All threads of the CTA call it;
// `tick` counts the tiles this CTA has done in this pass (the phases of its three barriers).
template <int D>
__device__ __noinline__ void sparse_careful_unit(const SparseCta<D>& c, const SparseGeom& g, const SparseUnits& s,
                                                 const SparseFwdArgs& a, const SparseMaps* maps, uint64_t* bars, int unit,
                                                 int warp, int lane, int& tick) {
  constexpr int kMmaWarp = 4 * kFwdGroups, kTmaWarp = 4 * kFwdGroups + 1;
  uint64_t *kv_full = bars, *s_done = bars + 1, *pv_done = bars + 2;
  const SparseUnit u(s, unit, a.heads, a.batch);
  const int grp = warp >> 2, r = (warp & 3) * 32 + lane;
  const bool softmax = warp < kMmaWarp;
  const uint32_t tmem_lane = c.tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
  const SparseRow<D> row(s, u, a, r);
  SparseStream st;
  if (warp == kTmaWarp) {
    st.start(s, a, unit, lane);
    st.open(g, s, a, lane);
  }
  if (softmax && grp < D / 64) row.stage_q(tmem_lane + kFwdColQ, grp, lane);
  float m_run = -INFINITY, l_run = 0.f;
  float* slot = c.smax;
  for (bool first = true;; first = false, ++tick) {
    bool last = false;
    if (warp == kTmaWarp) {
      uint32_t valid;
      last = next_tile(g, st.w, st.h, st.b, st.bx, c.source, valid);
      if (lane == 0) {
        c.desc[0].valid = valid;
        c.desc[0].flags = last ? kTileLast : 0u;
        if (!*c.abort_flag) {
          mbar_arrive_expect_tx(kv_full, 2 * sparse_tile_bytes<D>(g));
          load_sparse_tile<D>(c.sK, &maps->kx, &maps->kc, kv_full, c.source, g);
          load_sparse_tile<D>(c.sV, &maps->vx, &maps->vc, kv_full, c.source, g);
        }
      }
    }
    tc_fence_before_sync();
    // descriptor written; Q staged; the tile before is done with S and P.  Once a wait has run out, all leave together.
    if (__syncthreads_or(*c.abort_flag)) break;
    tc_fence_after_sync();
    last = reinterpret_cast<const volatile TileDesc*>(c.desc)->flags & kTileLast;
    const uint32_t valid4 = reinterpret_cast<const volatile TileDesc*>(c.desc)->valid;
    if (warp == kMmaWarp && lane == 0) {
      mbar_wait_spin(kv_full, tick & 1, c.abort_flag);
      tc_fence_after_sync();
      sparse_s<D>(c.tmem_base + kFwdColS, c.tmem_base + kFwdColQ, desc_kmajor(smem_u32(c.sK)));
      mma_commit(s_done);
    }
    if (softmax) {
      const int valid = (valid4 >> (8 * grp)) & 0xff;
      const uint32_t colS = tmem_lane + kFwdColS + grp * kFwdCols;
      mbar_wait(s_done, tick & 1, c.abort_flag);
      tc_fence_after_sync();
      uint32_t sv[32], pk[16];
      tmem_ld32(colS, sv);
      tmem_wait_ld();
      float mx = row_max(sv, valid);
      slot[grp * kTile + r] = mx;
      named_barrier_sync(1 + (warp & 3), 32 * kFwdGroups);
#pragma unroll
      for (int og = 0; og < kFwdGroups; ++og) mx = fmaxf(mx, slot[og * kTile + r]);
      const float m_new = fmaxf(m_run, mx * a.scale_log2);   // -inf while no key has a finite score
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m_use);
      m_run = m_new;
      l_run = l_run * alpha + sparse_exp32(sv, valid, a.scale_log2, -m_use, pk);
      tmem_st16(colS, pk);
      if (!first) {   // O is at rest: the P V of the tile before was awaited
#pragma unroll
        for (int c4 = 0; c4 < D / 32; ++c4) {
          if (c4 % kFwdGroups != grp) continue;
          tmem_ld32(tmem_lane + kFwdColO + c4 * 32, sv);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) sv[e] = __float_as_uint(__uint_as_float(sv[e]) * alpha);
          tmem_st32(tmem_lane + kFwdColO + c4 * 32, sv);
        }
      }
      tmem_wait_st();
    }
    tc_fence_before_sync();
    __syncthreads();   // P and the rescaled O are in tensor memory
    tc_fence_after_sync();
    if (warp == kMmaWarp && lane == 0) {
      sparse_pv<D>(c.tmem_base, c.tmem_base + kFwdColS, smem_u32(c.sV), first ? 0u : 1u);
      mma_commit(pv_done);
    }
    mbar_wait(pv_done, tick & 1, c.abort_flag);   // K, V, S, P and the descriptor may be overwritten
    tc_fence_after_sync();
    if (last) { ++tick; break; }   // the same for every thread
  }
  __syncthreads();
  if (softmax) {
    slot[grp * kTile + r] = l_run;
    named_barrier_sync(1 + (warp & 3), 32 * kFwdGroups);
    float l = 0.f;
#pragma unroll
    for (int og = 0; og < kFwdGroups; ++og) l += slot[og * kTile + r];
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint64_t chk2 = f32x2(0.f, 0.f);
    for (int c4 = grp; c4 < D / 32; c4 += kFwdGroups) {
      uint32_t acc[32];
      tmem_ld32(tmem_lane + kFwdColO + c4 * 32, acc);
      tmem_wait_ld();
      row.store(acc, inv, chk2, c4 * 32, lane);
    }
    if (grp == 0) row.store_lse(m_run, l);
  }
  tc_fence_before_sync();
  __syncthreads();   // the exchange slots and O may be overwritten
  tc_fence_after_sync();
}

// ---------------------------------------------------------------------------------- kernel
// grid.x CTAs share the units (at most kFwdMaxUnits each): CTA i takes units i, i + grid.x, ...
template <int D>
__global__ void __launch_bounds__(kSparseThreads, 1)
sparse_attn_fwd_kernel(const __grid_constant__ SparseMaps maps, const __grid_constant__ SparseFwdArgs a,
                       const __grid_constant__ SparseGeom g, const __grid_constant__ SparseUnits units_in) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align_1024(smem_raw);
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(smem + SparseFwdSmem<D>::kBars);
  const SparseBars bar(bar_mem);
  uint64_t* careful_bars = bar_mem + kSparseBarSlots;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(bar_mem + 48);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr uint32_t kTmemCols = 512;
  constexpr int kMmaWarp = 4 * kFwdGroups, kTmaWarp = 4 * kFwdGroups + 1;   // kTmaWarp: lists
  constexpr int kKWarp = kSparseThreads / 32 - 2, kVWarp = kSparseThreads / 32 - 1;

  SparseCta<D> c;
  c.sK = smem + SparseFwdSmem<D>::kK;
  c.sV = smem + SparseFwdSmem<D>::kV;
  c.smax = reinterpret_cast<float*>(smem + SparseFwdSmem<D>::kMax);
  c.desc = reinterpret_cast<TileDesc*>(smem + SparseFwdSmem<D>::kDesc);
  c.source = reinterpret_cast<TileSource*>(smem + SparseFwdSmem<D>::kSource);
  c.redo = reinterpret_cast<uint32_t*>(smem + SparseFwdSmem<D>::kRedo);
  c.abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  SparseUnits s = units_in;
  s.first = blockIdx.x;
  s.stride = gridDim.x;

  // the first list's entries are on their way while barriers and tensor memory are set up
  SparseStream stream;
  if (warp == kTmaWarp) stream.start(s, a, s.first, lane);
  if (warp == kKWarp && lane == 0) {
    tma_prefetch_desc(&maps.kx); tma_prefetch_desc(&maps.vx); tma_prefetch_desc(&maps.kc); tma_prefetch_desc(&maps.vc);
  }
  if (tid < kSparseBarSlots + 3) {   // the three of the careful pass behind them
    const int arrivals = tid < kSparseBarSlots ? SparseBars::arrivals(tid) : 1;
    if (arrivals > 0) mbar_init(bar_mem + tid, arrivals);
    fence_mbar_init();
  }
  if (tid == 0) *c.abort_flag = 0;
  if (tid < kFwdMaxUnits / 32) c.redo[tid] = 0;
  zero_uncovered_rows<D>(c.sK, kFwdKStages, g, tid, kSparseThreads);
  zero_uncovered_rows<D>(c.sV, kFwdVStages, g, tid, kSparseThreads);
  fence_proxy_async_smem();
  if (warp == kMmaWarp) {
    tmem_alloc(tmem_holder, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  c.tmem_base = *tmem_holder;
  dependents_may_start();

  bool asked = a.careful != 0;
  if (!a.careful) {
    if (warp == kTmaWarp) sparse_walk<D>(c, g, s, a, bar, stream, lane);
    else if (warp == kKWarp) { if (lane == 0) sparse_load_k<D>(c, g, maps, bar); }
    else if (warp == kVWarp) { if (lane == 0) sparse_load_v<D>(c, g, maps, bar); }
    else if (warp == kMmaWarp) { if (lane == 0) sparse_issue<D>(c, bar); }
    else if (warp < kMmaWarp) asked = sparse_softmax<D>(c, bar, warp, tid & 127, a.scale_log2);
    else asked = sparse_epilogue<D>(c, s, a, bar, warp, lane);
  }
  // every MMA of the fast pass has finished by now: the epilogue warps waited for the last one
  tc_fence_before_sync();
  if (__syncthreads_or(asked)) {
    int n = 0, tick = 0;
    for (int unit = s.first; unit < s.total; unit += s.stride, ++n) {
      tc_fence_before_sync();
      __syncthreads();
      tc_fence_after_sync();
      if (*c.abort_flag) break;
      if (!a.careful && !((c.redo[n >> 5] >> (n & 31)) & 1u)) continue;
      sparse_careful_unit<D>(c, g, s, a, &maps, careful_bars, unit, warp, lane, tick);
    }
  }
  settle_after_abort(c.abort_flag);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) tmem_dealloc(c.tmem_base, kTmemCols);
}

// Joins the parts of split units: weights exp(LSE_s - LSE), a warp per (sample, head, query) row.  Bandwidth: the parts are
// read once.  This kernel may be running while the one that writes the parts still does, so they are no read-only data to it:
// no const __restrict__, which would allow loads ahead of dependency_wait.
template <int D>
__global__ void __launch_bounds__(256)
sparse_combine_kernel(const float* part_o, const float* part_lse, const int splits, const long long rows, const int n_q,
                      const int heads, __nv_bfloat16* o, float* lse) {
  constexpr int kPer = D / 32;
  dependency_wait();
  const long long at = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (at >= rows) return;
  float top = -INFINITY;
  for (int i = 0; i < splits; ++i) top = fmaxf(top, part_lse[i * rows + at]);
  const float ref = top == -INFINITY ? 0.f : top;
  float total = 0.f, acc[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) acc[e] = 0.f;
  for (int i = 0; i < splits; ++i) {
    const float w = expf(part_lse[i * rows + at] - ref);   // 0 for a part without keys
    total += w;
    const float* src = part_o + (i * rows + at) * D + lane * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = fmaf(w, src[e], acc[e]);
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  const long long bh = at / n_q;
  const int i = static_cast<int>(at - bh * n_q), h = static_cast<int>(bh % heads);
  __nv_bfloat16* dst = o + (((bh / heads) * n_q + i) * heads + h) * D + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; e += 2) *reinterpret_cast<uint32_t*>(dst + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
  if (lane == 0 && lse != nullptr) lse[at] = total == 0.f ? -INFINITY : ref + logf(total);
}

}  // namespace astro
