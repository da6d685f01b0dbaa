// Choice of key blocks by a cheap score.
//   mean_j  = (sum over the tokens t of block j of k_t) / (tokens of block j), summed in fp64, kept in fp32
//   score_ij = mean of query block i . mean_j, in fp64
// and per query block the n_select largest scores.  A choice is a comparison: two scores that are equal or nearly so
// should come out in the same order whatever the order of the sums, so sums and products are fp64 and only the means are rounded,
// once, to fp32.  The fp64 sum of a block of up to 128 bf16 values is exact while their exponents lie within 38 binades (53 bits,
// less the 8 of a value and 7 of carries).  Values further apart leave rounding in its last bits, which depends on how many warps
// share a block, that is on the size of the launch: the fp32 mean can then differ by its last bit between a launch over a few
// frames and one over all.  Equal scores go to the lower block, NaN ranks below everything.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "attn_common.cuh"

namespace astro {

// Key blocks of one call: `ctx` blocks of the held cache frames (frame by frame in logical order: sink, then window
// oldest to newest; `per_frame` blocks of `block` tokens each, the last one shorter), then the chunk's own.
struct KeyBlocks {
  int block, per_frame, ctx, total;
  int tokens_per_frame, n_kc;
  int sink_held, sink_slots, win_head, win_slots;
};

__device__ __forceinline__ int key_block_slot(const KeyBlocks& kb, int frame) {
  if (frame < kb.sink_held) return frame;
  const int i = kb.win_head + (frame - kb.sink_held);
  return kb.sink_slots + (i >= kb.win_slots ? i - kb.win_slots : i);
}

// ------------------------------------------------------------------------------------------------ means
// Rows of one source of blocks: row t of (sample b, head h) starts at base + b * sb + h * sh + t * st (elements).
struct PoolSource {
  const __nv_bfloat16* base;
  long long sb, sh, st;
  float* out;              // [b][h][out_row][D]
  long long out_b, out_h;  // rows per sample, rows per head of `out`
  int tokens, block, blocks;
  double inv_block, inv_last;   // 1 / tokens of a full block, of the last one
};

constexpr int kPoolThreads = 256;
constexpr int kPoolBatch = 6;   // token rows a thread has in flight, twice (the next batch is asked for before this one is added)

// Adds N rows of 8 bf16 values to the sums.  Conversions to fp64 are what a pool spends most of its issue time on (14.6 us with
// one per value, 11.7 without the sums): two rows are added in fp32 first and converted together, 13.5.  Where that sum
// s = a + b is not exact the two are added one by one; it is exact if s - a gives b and s - b gives a back (the error term of
// the two-sum algorithm is then zero; an infinity or a NaN never gives both back, -0 does not always).  With exponents less than 16 apart it always is; of pairs of normal deviates one in
// 10^5 is not.
template <int N>
__device__ __forceinline__ void pool_add(const uint4 (&v)[N], double (&acc)[8]) {
  static_assert(N % 2 == 0, "pairs of rows");
  const uint64_t minus = f32x2(-1.f, -1.f);
#pragma unroll
  for (int u = 0; u < N; u += 2) {
    const uint32_t a[4] = {v[u].x, v[u].y, v[u].z, v[u].w}, b[4] = {v[u + 1].x, v[u + 1].y, v[u + 1].z, v[u + 1].w};
    float s[8];
    uint32_t off = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a0 = __uint_as_float(a[e] << 16), a1 = __uint_as_float(a[e] & 0xffff0000u);
      const float b0 = __uint_as_float(b[e] << 16), b1 = __uint_as_float(b[e] & 0xffff0000u);
      const uint64_t a2 = f32x2(a0, a1), b2 = f32x2(b0, b1), s2 = add2(a2, b2);
      float x0, x1, y0, y1;
      f32x2_split(fma2(a2, minus, s2), x0, x1);
      f32x2_split(fma2(b2, minus, s2), y0, y1);
      f32x2_split(s2, s[2 * e], s[2 * e + 1]);
      off |= __float_as_uint(x0) ^ __float_as_uint(b0);
      off |= __float_as_uint(x1) ^ __float_as_uint(b1);
      off |= __float_as_uint(y0) ^ __float_as_uint(a0);
      off |= __float_as_uint(y1) ^ __float_as_uint(a1);
    }
    if (off == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += static_cast<double>(s[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[2 * e] += static_cast<double>(__uint_as_float(a[e] << 16));
        acc[2 * e] += static_cast<double>(__uint_as_float(b[e] << 16));
        acc[2 * e + 1] += static_cast<double>(__uint_as_float(a[e] & 0xffff0000u));
        acc[2 * e + 1] += static_cast<double>(__uint_as_float(b[e] & 0xffff0000u));
      }
    }
  }
}

// A warp's part of the sum over the rows of one block: D/8 lanes side by side hold 8 elements each; the warp's lane groups
// take rows t, t + step, ...  On return every lane of a column has the warp's sum.
template <int D>
__device__ __forceinline__ void pool_rows(const __nv_bfloat16* src, long long st, int count, int t, int step, double (&acc)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  uint4 v[kPoolBatch];
  auto fetch = [&]() {
#pragma unroll
    for (int u = 0; u < kPoolBatch; ++u)
      v[u] = t + u * step < count ? __ldcs(reinterpret_cast<const uint4*>(src + (t + u * step) * st)) : make_uint4(0, 0, 0, 0);
  };
  fetch();
  while (t < count) {
    uint4 now[kPoolBatch];
#pragma unroll
    for (int u = 0; u < kPoolBatch; ++u) now[u] = v[u];
    t += kPoolBatch * step;
    fetch();
    pool_add(now, acc);
  }
  __syncwarp();
#pragma unroll
  for (int x = D / 8; x < 32; x *= 2)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], x);
}
__device__ __forceinline__ void store_mean(float* out, const double (&acc)[8], double inv) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = static_cast<float>(acc[e] * inv);
  reinterpret_cast<float4*>(out)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(out)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// The mean of one block by `share` neighbouring warps of a thread block: their
// partial sums are joined in shared memory by the first of them.  All threads of the thread block together.
template <int D>
__device__ __forceinline__ void pool_shared(const __nv_bfloat16* src, long long st, int count, bool there, int share, float* out,
                                            double inv, double (*part)[8][D / 8]) {
  constexpr int kCols = D / 8, kGroups = 32 / kCols;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = lane % kCols;
  double acc[8];
  pool_rows<D>(src + col * 8, st, count, (warp % share) * kGroups + lane / kCols, share * kGroups, acc);
  if (share > 1) {
    if (lane < kCols && warp % share) {
#pragma unroll
      for (int e = 0; e < 8; ++e) part[warp][e][col] = acc[e];
    }
    __syncthreads();
    if (warp % share == 0)
      for (int r = 1; r < share; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += part[warp + r][e][col];
  }
  if (there && lane < kCols && warp % share == 0) store_mean(out + col * 8, acc, inv);
}

// The means of cached blocks: `share` warps (1, 2, 4 or 8) per block of one head.  Everything is resident at once and every
// warp streams by itself: 58 MB in 13.5 us (a thread block per block, all its partial sums joined in shared memory, 17.2;
// bulk copies into a ring of pieces per warp, twice the bytes in flight, 14.6).
// grid.x * (8 / share) covers the `blocks` blocks of the frames from logical frame `frame0` on; grid.y = head, grid.z = sample.
template <int D>
__global__ void __launch_bounds__(kPoolThreads)
block_pool_kernel(const PoolSource s, const KeyBlocks kb, const int frame0, const int share) {
  const int unit = blockIdx.x * (blockDim.x / 32 / share) + (threadIdx.x >> 5) / share;
  const int f = unit / kb.per_frame, j = unit - f * kb.per_frame;
  const int h = blockIdx.y, b = blockIdx.z;
  const bool there = unit < s.blocks;
  const int slot = there ? key_block_slot(kb, frame0 + f) : 0;
  const int count = there ? min(s.block, s.tokens - j * s.block) : 0;
  __shared__ double part[kPoolThreads / 32][8][D / 8];
  pool_shared<D>(
      s.base + b * s.sb + h * s.sh + (static_cast<long long>(slot) * s.tokens + static_cast<long long>(j) * s.block) * s.st, s.st,
      count, there, share, s.out + (b * s.out_b + h * s.out_h + static_cast<long long>(slot) * kb.per_frame + j) * D,
      count == s.block ? s.inv_block : s.inv_last, part);
}

// The same for the blocks of two contiguous tensors (queries, chunk keys), numbered one after the other.
template <int D>
__global__ void __launch_bounds__(kPoolThreads)
block_mean_kernel(const PoolSource s0, const PoolSource s1, const int share) {
  dependents_may_start();
  const int unit = blockIdx.x * (blockDim.x / 32 / share) + (threadIdx.x >> 5) / share;
  const int h = blockIdx.y, b = blockIdx.z;
  const bool second = unit >= s0.blocks, there = unit < s0.blocks + s1.blocks;
  const PoolSource& s = second ? s1 : s0;
  const int j = second ? unit - s0.blocks : unit;
  const int count = there ? min(s.block, s.tokens - j * s.block) : 0;
  __shared__ double part[kPoolThreads / 32][8][D / 8];
  pool_shared<D>(s.base + b * s.sb + h * s.sh + static_cast<long long>(j) * s.block * s.st, s.st, count, there, share,
                               s.out + (b * s.out_b + h * s.out_h + j) * D, count == s.block ? s.inv_block : s.inv_last, part);
}

// ------------------------------------------------------------------------------------------------ choice
constexpr int kSelectThreads = 512;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kSelectRows = 8;     // query blocks of one MMA tile
constexpr int kSelectHeld = 16;    // keys a lane holds in registers

// A double as an unsigned integer of the same order; NaN becomes 0, below every number.
__device__ __forceinline__ unsigned long long order_key(double x) {
  if (x != x) return 0ull;
  const unsigned long long u = static_cast<unsigned long long>(__double_as_longlong(x + 0.0));   // -0 ranks as 0
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
constexpr unsigned long long kKeptKey = ~0ull;   // above the key of +infinity

struct SelectArgs {
  const float* pooled;    // [cache_batch][H][slots][per_frame][D]
  const float* q_mean;    // [B][H][q_blocks][D]
  const float* kc_mean;   // [B][H][chunk blocks][D]
  int* blocks;            // [B][H][q_blocks][n_select]
  int heads, q_blocks, n_select, cache_shared, keep_sink, keep_chunk;
  int rows;               // query blocks of a thread block, at most kSelectRows
};

// c[8 x 8] += a[8 x 4] b[4 x 8], fp64: lane holds a[lane / 4][lane % 4], b[lane % 4][lane / 4] and
// c[lane / 4][2 (lane % 4) + {0, 1}].
__device__ __forceinline__ void mma_f64(double (&c)[2], double a, double b) {
  asm("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};"
      : "+d"(c[0]), "+d"(c[1])
      : "d"(a), "d"(b));
}

// A warp's search for the cut between the `want` largest of `total` keys and the others.  The cut is the want-th largest key
// (the largest value that at least `want` keys reach) or any value that exactly `want` keys reach; `ties` is how many
// of the keys equal to it belong to the chosen ones.  count(p) counts the keys of a lane for which p holds; keys of 0 that
// pad a lane are not counted because a candidate is never 0.
template <typename Count>
__device__ __forceinline__ unsigned long long select_cut(int want, int total, int& ties, Count count) {
  unsigned long long cut = 0;
  int reach = total;
  for (int bit = 63; bit >= 0 && reach != want; --bit) {
    const unsigned long long cand = cut | (1ull << bit);
    const int n = __reduce_add_sync(0xffffffffu, count([&](unsigned long long x) { return x >= cand; }));
    if (n >= want) {
      cut = cand;
      reach = n;
    }
  }
  ties = total;
  if (reach != want) ties = want - __reduce_add_sync(0xffffffffu, count([&](unsigned long long x) { return x > cut; }));
  return cut;
}

// The thread blocks of grid.x share the query blocks of one head of one sample, `rows` (up to eight) at a time.  Scores: a
// warp per eight key blocks, fp64 MMAs over the head dimension; the contraction index is dealt to the lanes so that each
// reads 16 contiguous bytes of a row (the same order on both sides, so nothing else changes).  Then a warp per query block
// finds the n-th largest key bit by bit, stopping as soon as a candidate separates exactly n, and writes the blocks above
// it, and as many equal to it as there is room for, in order.  Scores by fused multiply-adds and shuffles, a warp per key
// block, took 42 us for a chunk of 37 x 12 query blocks and 273 key blocks; by MMAs 8.
// share > 0: the kernel first works out the means of the head's query blocks and chunk blocks itself, `share` warps each, and
// grid.x is one cluster, whose barrier makes them known.  For the single query this saves a launch (13.2 us against
// 16.3); the 76 blocks of a chunk's queries and keys want more SMs than the clusters have (23.9 us against 21.9), so there
// they come from block_mean_kernel, and this kernel is launched as its dependent with share = 0.
// Dynamic shared memory: keys [rows][total].
template <int D>
__global__ void __launch_bounds__(kSelectThreads)
block_select_kernel(const SelectArgs a, const KeyBlocks kb, const PoolSource qs, const PoolSource ks, const int share) {
  extern __shared__ unsigned long long s_key[];
  constexpr int kSteps = D / 16;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = blockIdx.y, b = blockIdx.z, rank = blockIdx.x, size = gridDim.x;
  if (share == 0) {
    dependency_wait();
  } else {
    __shared__ double part[kSelectWarps][8][D / 8];
    const int per_pass = kSelectWarps / share, units = qs.blocks + ks.blocks;
    for (int u0 = rank * per_pass; u0 < units; u0 += size * per_pass) {   // the same for the whole thread block
      const int unit = u0 + warp / share;
      const bool there = unit < units, second = unit >= qs.blocks;
      const PoolSource& s = second ? ks : qs;
      const int j = second ? unit - qs.blocks : unit;
      const int count = there ? min(s.block, s.tokens - j * s.block) : 0;
      pool_shared<D>(s.base + b * s.sb + h * s.sh + static_cast<long long>(j) * s.block * s.st, s.st, count, there, share,
                                     s.out + (b * s.out_b + h * s.out_h + j) * D, count == s.block ? s.inv_block : s.inv_last, part);
      __syncthreads();   // the parts have been read
    }
    __syncwarp();
    cluster_sync_all();
  }
  const int slots = kb.sink_slots + kb.win_slots, chunk_blocks = kb.total - kb.ctx;
  const float* ctx = a.pooled + static_cast<long long>(a.cache_shared ? 0 : b) * a.heads * slots * kb.per_frame * D +
                     static_cast<long long>(h) * slots * kb.per_frame * D;
  const float* own = a.kc_mean + (static_cast<long long>(b) * a.heads + h) * chunk_blocks * D;
  const int pair = lane >> 2, col = (lane & 3) * 4;
  for (int q0 = rank * a.rows; q0 < a.q_blocks; q0 += size * a.rows) {
    const int rows = min(a.rows, a.q_blocks - q0);
    float4 q[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      q[i] = pair < rows ? *reinterpret_cast<const float4*>(
                               a.q_mean + ((static_cast<long long>(b) * a.heads + h) * a.q_blocks + q0 + pair) * D + i * 16 + col)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int j0 = warp * 8; j0 < kb.total; j0 += kSelectWarps * 8) {
      const int j = j0 + pair;
      const float* src = nullptr;
      if (j < kb.ctx) {
        const int f = j / kb.per_frame;
        src = ctx + (static_cast<long long>(key_block_slot(kb, f)) * kb.per_frame + (j - f * kb.per_frame)) * D;
      } else if (j < kb.total) {
        src = own + static_cast<long long>(j - kb.ctx) * D;
      }
      float4 k[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        k[i] = src ? *reinterpret_cast<const float4*>(src + i * 16 + col) : make_float4(0.f, 0.f, 0.f, 0.f);
      double even[2] = {0.0, 0.0}, odd[2] = {0.0, 0.0};   // two chains
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        mma_f64(even, q[i].x, k[i].x);
        mma_f64(odd, q[i].y, k[i].y);
        mma_f64(even, q[i].z, k[i].z);
        mma_f64(odd, q[i].w, k[i].w);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int to = j0 + 2 * (lane & 3) + e;
        if (pair < rows && to < kb.total) {
          const bool keep = to < kb.ctx ? a.keep_sink && to < kb.sink_held * kb.per_frame : a.keep_chunk != 0;
          s_key[static_cast<long long>(pair) * kb.total + to] = keep ? kKeptKey : order_key(even[e] + odd[e]);
        }
      }
    }
    __syncthreads();
    for (int r = warp; r < rows; r += kSelectWarps) {
      const unsigned long long* key = s_key + static_cast<long long>(r) * kb.total;
      int* out = a.blocks + ((static_cast<long long>(b) * a.heads + h) * a.q_blocks + q0 + r) * a.n_select;
      const int want = min(a.n_select, kb.total);
      int ties;
      unsigned long long cut;
      // up to 512 keys sit in the lanes' registers during the search, more are read again for every bit
      if (kb.total <= 32 * kSelectHeld) {
        unsigned long long held[kSelectHeld];
#pragma unroll
        for (int i = 0; i < kSelectHeld; ++i) held[i] = lane + 32 * i < kb.total ? key[lane + 32 * i] : 0ull;
        cut = select_cut(want, kb.total, ties, [&](auto reaches) {
          int n = 0;
#pragma unroll
          for (int i = 0; i < kSelectHeld; ++i) n += reaches(held[i]) ? 1 : 0;
          return n;
        });
      } else {
        cut = select_cut(want, kb.total, ties, [&](auto reaches) {
          int n = 0;
          for (int j = lane; j < kb.total; j += 32) n += reaches(key[j]) ? 1 : 0;
          return n;
        });
      }
      int at = 0;
      for (int j0 = 0; j0 < kb.total; j0 += 32) {
        const int j = j0 + lane;
        const unsigned long long x = j < kb.total ? key[j] : 0ull;
        const bool equal = j < kb.total && x == cut;
        const unsigned eq = __ballot_sync(0xffffffffu, equal);
        const bool take = (j < kb.total && x > cut) || (equal && __popc(eq & ((1u << lane) - 1u)) < ties);
        ties = max(0, ties - __popc(eq));
        const unsigned mask = __ballot_sync(0xffffffffu, take);
        if (take) out[at + __popc(mask & ((1u << lane) - 1u))] = j;
        at += __popc(mask);
      }
      for (int i = want + lane; i < a.n_select; i += 32) out[i] = -1;
    }
    __syncthreads();   // the keys have been read
  }
}

}  // namespace astro
