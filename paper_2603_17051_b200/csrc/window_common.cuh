// Attention of whole sequences in which a query sees its own block of tokens, a window in front of it and the first tokens
// (sinks): what the kernels share about who sees whom.
//
// With c = i / block, query i sees key j < len iff j < min(len, (c+1) block) and (j < sink or j >= (c+1) block - window).
// window >= block, so every query sees itself.  Queries from len on see nothing.
//
// Queries and keys are cut into tiles of 128 on one grid.  A query tile's keys are the tiles [0, a1) of the sinks and [w0, w1)
// of the window (a1 = w0 = 0 where they meet); its own tile, the diagonal one, lies in the second.  A pair of tiles is full when every
// live row sees every key; the others are masked bit by bit.
#pragma once
#include "attn_common.cuh"

namespace astro {

// A divisor that a whole launch shares: quotients of 0 <= x < 2^31 by one wide multiplication (Granlund and Montgomery, "Division by
// invariant integers using multiplication", 1994).  With l = ceil(log2 d) and mul = floor(2^32 (2^l - d) / d) + 1 the quotient is
// (floor(mul x / 2^32) + x) / 2^l.  A kernel's start is a chain of such quotients: with the operator's some 150 clocks each, a
// dK/dV CTA took 2300 to its first barrier.
struct Divisor {
  int d, shift;
  uint32_t mul;
  __host__ void set(int d_) {
    d = d_;
    shift = 0;
    while ((1u << shift) < static_cast<uint32_t>(d)) ++shift;
    mul = static_cast<uint32_t>((((1ull << shift) - d) << 32) / d + 1);
  }
  __host__ __device__ __forceinline__ int quot(int x) const {
#ifdef __CUDA_ARCH__
    const uint32_t high = __umulhi(mul, static_cast<uint32_t>(x));
#else
    const uint32_t high = static_cast<uint32_t>((static_cast<unsigned long long>(mul) * static_cast<uint32_t>(x)) >> 32);
#endif
    return static_cast<int>((high + static_cast<uint32_t>(x)) >> shift);
  }
};

struct WinMask {
  int n, window, sink;   // window <= n + block, sink <= n
  Divisor block;         // <= n
  const int* lengths;           // may be null: n each
  __host__ __device__ __forceinline__ int length(int b) const { return lengths == nullptr ? n : max(0, min(n, lengths[b])); }
  // the keys of query i of a sequence of `len`: [0, sink) below hi, and [lo, hi)
  __host__ __device__ __forceinline__ void keys_of(int i, int len, int& lo, int& hi) const {
    const int end = (block.quot(i) + 1) * block.d;
    lo = max(0, end - window);
    hi = min(len, end);
  }
  // Whether query i sees one key alone, which is itself: its weight is 1 whatever the scores, and dS is 0.
  __device__ __forceinline__ bool one_key(int i, int len) const {
    int lo, hi;
    keys_of(i, len, lo, hi);
    return hi - lo + min(sink, lo) == 1;
  }
  // the queries of key j: [first, last)
  __host__ __device__ __forceinline__ void queries_of(int j, int len, int& first, int& last) const {
    first = block.quot(j) * block.d;
    last = j < sink ? len : min(len, block.quot(j + window) * block.d);
  }
};

// 32 columns from `base` on: the bits of those below `end` (or all, or none).
__host__ __device__ __forceinline__ uint32_t bits_below(int end, int base) {
  const int x = end - base;
  return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u;
}

// The key tiles of a query tile.
struct WinTiles {
  int a1, w0, w1;        // [0, a1) and [w0, w1)
  int full_sink, full_lo, full_hi;   // full: tiles below full_sink, and [full_lo, full_hi)
  // a query tile that starts at row i0 < len
  __host__ __device__ __forceinline__ void set(const WinMask& m, int i0, int len) {
    int lo_min, lo_max, hi_min, hi_max;
    m.keys_of(i0, len, lo_min, hi_min);
    m.keys_of(min(i0 + kTile, len) - 1, len, lo_max, hi_max);
    w0 = lo_min / kTile;
    w1 = (hi_max + kTile - 1) / kTile;
    a1 = (min(m.sink, hi_max) + kTile - 1) / kTile;
    if (a1 >= w0) a1 = w0 = 0;
    const int sink_min = min(m.sink, hi_min);
    full_sink = sink_min / kTile;
    full_lo = lo_max <= sink_min ? 0 : (lo_max + kTile - 1) / kTile;
    full_hi = hi_min / kTile;
  }
  __host__ __device__ __forceinline__ int count() const { return a1 + w1 - w0; }
  __host__ __device__ __forceinline__ int first() const { return a1 > 0 ? 0 : w0; }
  __host__ __device__ __forceinline__ int next(int tile) const { return tile + 1 == a1 ? w0 : tile + 1; }   // from w1 on: none left
  __host__ __device__ __forceinline__ bool full(int tile) const { return tile < full_sink || (tile >= full_lo && tile < full_hi); }
  // where the run of full tiles that `tile` is in ends
  __host__ __device__ __forceinline__ int run_end(int tile) const {
    int e = full_hi;
    if (tile < full_sink && !(full_lo <= full_sink && full_hi > full_sink)) e = full_sink;
    return tile < a1 ? min(e, a1) : min(e, w1);
  }
};

// Work in the order in which CTAs take it: `lists` (sample, head) lists of `tiles` tiles each.  Tile by tile over all lists the
// long ones come first and the end is even; list by list the CTAs that run together share K and V in L2 (5 % on a video's 12 lists of
// 256 tiles).  So: groups of lists of one size, one after the other, tile by tile within, eight rounds of 148 CTAs and more in each.
struct WinOrder {
  int lists, tiles, per_group;
  Divisor group_tiles, by_lists, by_rest;   // a group's tiles; its lists, the last group's
  __host__ void set(int lists_, int tiles_) {
    lists = lists_;
    tiles = tiles_;
    const long long groups = static_cast<long long>(lists) * tiles / (8 * 148);
    per_group = groups <= 1 ? lists : static_cast<int>((lists + groups - 1) / groups);
    group_tiles.set(max(1, static_cast<int>(min(static_cast<long long>(per_group) * tiles, 0x40000000ll))));
    by_lists.set(per_group);
    by_rest.set(lists - (lists - 1) / per_group * per_group);
  }
  __device__ __forceinline__ void place(int i, int& tile, int& list) const {
    const int first = group_tiles.quot(i) * per_group;
    i -= first * tiles;
    const bool rest = first + per_group > lists;
    tile = rest ? by_rest.quot(i) : by_lists.quot(i);
    list = first + i - tile * (rest ? by_rest.d : by_lists.d);
  }
};

struct WinStrides {
  long long b, t, h;     // in elements
};

// The four rows of a lane's quad in a strided tensor (see QuadRows).
__device__ __forceinline__ QuadRows quad_rows_strided(const __nv_bfloat16* base, const WinStrides& s, int b, int h, int n_rows,
                                                      int own_row) {
  QuadRows q;
  const int row_first = own_row & ~3;
  q.stride = static_cast<size_t>(s.t);
  q.first = const_cast<__nv_bfloat16*>(base) + b * s.b + row_first * s.t + h * s.h;
  q.valid = n_rows - row_first;
  return q;
}

// Rows [first_row, 128) of a tile that a bulk copy has brought become zeros.  A whole warp, behind its wait for the copy.
template <int D>
__device__ __forceinline__ void zero_rows_by_warp(uint8_t* smem_tile, int first_row, int lane) {
  const int pieces = (kTile - first_row) * 8 * TileGeom<D>::kBlocks;
  for (int i = lane; i < pieces; i += 32) {
    const int blk = i % TileGeom<D>::kBlocks, x = i / TileGeom<D>::kBlocks;
    *reinterpret_cast<uint4*>(smem_tile + blk * TileGeom<D>::kBlockBytes + first_row * 128 + x * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

}  // namespace astro
