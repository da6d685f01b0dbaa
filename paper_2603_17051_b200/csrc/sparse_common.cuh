// Shared pieces of the attention kernels that walk over lists of key blocks: how a list becomes a stream of key tiles.
//
// A key tile is the 128 keys of one MMA.  Blocks of up to 32, 64 or 128 tokens take a quarter, half or all of it (their
// `pad` rows; a tile then holds 128 / pad blocks).  One TMA box is one block: `block` rows by 64 columns, out of a 5-D
// map {d, token of the frame, slot, head, batch} whose second extent ends with the frame (or the chunk), so that what
// a short last block lacks is filled with zeros, never with a neighbouring slot's stale bytes.  The rows between
// `block` and `pad` are zeroed once per kernel and never written again.  So every row of a tile that is no key of
// the list is zero in shared memory; its scores are masked as well.  A part of a tile for which the list has no block left is
// loaded from behind the end of the tensor (all zeros).
#pragma once
#include "attn_common.cuh"
#include "block_select.cuh"

namespace astro {

constexpr int kSpParts = 4;        // most blocks of a tile
constexpr int kSpDescs = 8;        // tile descriptors in flight (a power of two; the streams look two tiles ahead)

// How a block size fills a tile.
struct SparseGeom {
  KeyBlocks kb;
  int pad, per_tile;
  int chunk_fill;   // 1: rows of zeros are loaded from behind the chunk, 0: from behind a cache frame
};
__host__ __device__ inline int sparse_pad(int block) { return block <= 32 ? 32 : block <= 64 ? 64 : 128; }

// A block of a list: where its tokens are.
struct BlockRef {
  int row0, slot, valid, chunk;
};
__device__ __forceinline__ BlockRef block_ref(const SparseGeom& g, int id) {
  BlockRef r;
  if (id < g.kb.ctx) {
    const int f = id / g.kb.per_frame;
    r.row0 = (id - f * g.kb.per_frame) * g.kb.block;
    r.slot = key_block_slot(g.kb, f);
    r.valid = min(g.kb.block, g.kb.tokens_per_frame - r.row0);
    r.chunk = 0;
  } else {
    r.row0 = (id - g.kb.ctx) * g.kb.block;
    r.slot = 0;
    r.valid = min(g.kb.block, g.kb.n_kc - r.row0);
    r.chunk = 1;
  }
  return r;
}

// What the other roles are told about tile J of a stream (descriptor J % kSpDescs in shared memory).
struct TileDesc {
  uint32_t valid;   // byte g: valid keys of key group g (32 keys each)
  uint32_t flags;
};
constexpr uint32_t kTileThere = 1u, kTileFirst = 2u, kTileLast = 4u, kTileEnd = 8u;   // first / last of its unit; last of all
constexpr int kTileLiveShift = 8;   // bits 8..10: quarters (32 rows) of the query tile that hold a query, 1..4
__device__ __forceinline__ uint32_t live_quarters(int n_q, int qt) { return (min(kTile, n_q - qt * kTile) + 31) / 32; }

// Where the producer finds the blocks of a tile.
struct TileSource {
  BlockRef part[kSpParts];
  int h, b, bx;   // head, sample of the chunk tensors, sample of the cache
};

// Walks over one list of block ids, 32 entries at a time; the next 32 are fetched while these are used.  Entries that
// name no block are skipped.  All lanes of a warp together.
struct ListWalker {
  const int* list;
  int n, pos, lane, ahead;
  uint32_t mask;
  BlockRef ref;
  __device__ void fetch(const SparseGeom& g) {
    while (mask == 0 && pos < n) {
      const int id = ahead;
      pos += 32;
      ahead = pos + lane < n ? list[pos + lane] : -1;
      const bool ok = id >= 0 && id < g.kb.total;
      mask = __ballot_sync(0xffffffffu, ok);
      if (ok) ref = block_ref(g, id);
    }
  }
  // Opens a list whose first 32 entries have been asked for before (first_entries).
  __device__ void open(const SparseGeom& g, const int* entries, int count, int lane_, int first) {
    list = entries;
    n = count;
    pos = 0;
    lane = lane_;
    mask = 0;
    ahead = first;
    fetch(g);
  }
  static __device__ int first_entries(const int* entries, int count, int lane) { return lane < count ? entries[lane] : -1; }
  __device__ bool done() const { return mask == 0; }
  __device__ BlockRef take(const SparseGeom& g) {
    const int from = __ffs(mask) - 1;
    BlockRef r;
    r.row0 = __shfl_sync(0xffffffffu, ref.row0, from);
    r.slot = __shfl_sync(0xffffffffu, ref.slot, from);
    r.valid = __shfl_sync(0xffffffffu, ref.valid, from);
    r.chunk = __shfl_sync(0xffffffffu, ref.chunk, from);
    mask &= mask - 1;
    fetch(g);
    return r;
  }
};

// The next tile of a list into a source and a descriptor (written by lane 0); returns whether it is the list's last.
// An empty list makes one tile of zeros without a valid key, so that every unit has a tile.
__device__ __forceinline__ bool next_tile(const SparseGeom& g, ListWalker& w, int h, int b, int bx, TileSource* src,
                                          uint32_t& valid) {
  valid = 0;
  for (int p = 0; p < g.per_tile; ++p) {
    BlockRef r;
    if (!w.done()) {
      r = w.take(g);
    } else {
      r.row0 = g.chunk_fill ? g.kb.n_kc : g.kb.tokens_per_frame;   // every row of the box is behind the end
      r.slot = 0;
      r.valid = 0;
      r.chunk = g.chunk_fill;
    }
    if (w.lane == 0) src->part[p] = r;
    for (int k = 0; k < g.pad; k += 32) {
      const int v = r.valid - k;
      valid |= static_cast<uint32_t>(v < 0 ? 0 : v > 32 ? 32 : v) << (8 * ((p * g.pad + k) / 32));
    }
  }
  if (w.lane == 0) { src->h = h; src->b = b; src->bx = bx; }
  return w.done();
}

// One arrival for the whole warp, behind everything its lanes have done: 16 arrivals per key tile instead of 512 on one
// barrier (they are served one by one).
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void warp_arrive_at(uint32_t bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive_at(bar);
}

struct SparseMaps {
  CUtensorMap kx, vx, kc, vc;
};

// One operand of a tile; `ctx` and `chunk` are its two maps.  One thread.
template <int D>
__device__ __forceinline__ void load_sparse_tile(uint8_t* smem_tile, const CUtensorMap* ctx, const CUtensorMap* chunk,
                                                 uint64_t* bar, const TileSource* src, const SparseGeom& g) {
  for (int p = 0; p < g.per_tile; ++p) {
    const BlockRef r = src->part[p];
    const CUtensorMap* tm = r.chunk ? chunk : ctx;
    const int bb = r.chunk ? src->b : src->bx;
#pragma unroll
    for (int blk = 0; blk < TileGeom<D>::kBlocks; ++blk)
      tma_load_5d(smem_tile + blk * TileGeom<D>::kBlockBytes + p * g.pad * 128, tm, bar, blk * 64, r.row0, r.slot, src->h, bb);
  }
}
template <int D> __device__ __forceinline__ uint32_t sparse_tile_bytes(const SparseGeom& g) {
  return static_cast<uint32_t>(g.per_tile * g.kb.block * 128 * TileGeom<D>::kBlocks);
}

// Zeroes the rows of `tiles` consecutive tiles that no box covers.  All threads of the CTA; the caller publishes it to
// the async proxy.
template <int D>
__device__ __forceinline__ void zero_uncovered_rows(uint8_t* smem_tiles, int tiles, const SparseGeom& g, int tid, int threads) {
  const int gap = g.pad - g.kb.block;
  const int rows = tiles * TileGeom<D>::kBlocks * g.per_tile * gap;
  for (int i = tid; i < rows * 8; i += threads) {
    const int row = i >> 3, piece = row / gap, in_gap = row - piece * gap;
    const int block = piece / g.per_tile, p = piece - block * g.per_tile;
    *reinterpret_cast<uint4*>(smem_tiles + block * TileGeom<D>::kBlockBytes + (p * g.pad + g.kb.block + in_gap) * 128 + (i & 7) * 16) =
        make_uint4(0, 0, 0, 0);
  }
}

}  // namespace astro
