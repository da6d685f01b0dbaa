// Choice of key blocks by a cheap score.
//   mean_j  = (sum over the tokens t of block j of k_t) / (tokens of block j), summed in fp64, kept in fp32
//   score_ij = mean of query block i . mean_j, in fp64
// and per query block the n_select largest scores.  A choice is a comparison: two scores that are equal or nearly so
// must come out in the same order whatever the order of the sums, so sums and products are fp64 (the sum of a block
// of bf16 values is exact there) and only the means are rounded, once, to fp32.  Equal scores go to the lower block,
// NaN ranks below everything.
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
};

constexpr int kPoolThreads = 256;

// One block of tokens of one head per thread block: D/8 threads side by side hold 8 elements each, the others walk the
// tokens; partial sums meet in shared memory.  Bandwidth bound: every token row is read once, 16 bytes per thread.
// grid.x = blocks of source 0, then of source 1 (n0 of the first); grid.y = head, grid.z = sample.
// `frames` > 0: source 0 is the cache storage, and grid.x walks frames x per_frame blocks from logical frame `frame0`.
template <int D>
__global__ void __launch_bounds__(kPoolThreads)
block_pool_kernel(const PoolSource s0, const PoolSource s1, const int n0, const KeyBlocks kb, const int frame0,
                  const int cache_source) {
  constexpr int kCols = D / 8, kRows = kPoolThreads / kCols;
  const bool second = static_cast<int>(blockIdx.x) >= n0;
  const PoolSource& s = second ? s1 : s0;
  int j = second ? blockIdx.x - n0 : blockIdx.x;
  const int h = blockIdx.y, b = blockIdx.z;
  long long first_row = 0, out_row = j;
  if (cache_source) {
    const int f = j / kb.per_frame, slot = key_block_slot(kb, frame0 + f);
    j -= f * kb.per_frame;
    first_row = static_cast<long long>(slot) * s.tokens;
    out_row = static_cast<long long>(slot) * kb.per_frame + j;
  }
  const int count = min(s.block, s.tokens - j * s.block);
  const int col = threadIdx.x % kCols, row = threadIdx.x / kCols;
  const __nv_bfloat16* src = s.base + b * s.sb + h * s.sh + (first_row + static_cast<long long>(j) * s.block) * s.st + col * 8;
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
#pragma unroll 4
  for (int t = row; t < count; t += kRows) {
    const uint4 v = *reinterpret_cast<const uint4*>(src + t * s.st);
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __bfloat1622float2(p[e]);
      acc[2 * e] += static_cast<double>(f.x);
      acc[2 * e + 1] += static_cast<double>(f.y);
    }
  }
  __shared__ double part[kRows][D + 2];
#pragma unroll
  for (int e = 0; e < 8; ++e) part[row][col * 8 + e] = acc[e];
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kPoolThreads) {
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) sum += part[r][e];
    s.out[((b * s.out_b + h * s.out_h) + out_row) * D + e] = static_cast<float>(sum / static_cast<double>(count));
  }
}

// ------------------------------------------------------------------------------------------------ choice
constexpr int kSelectThreads = 256;
constexpr int kSelectWarps = kSelectThreads / 32;

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
};

// R query blocks of one head per thread block: the key means are read once for all R.  Scores: a warp per key block,
// D/32 elements per lane, fp64 fused multiply-adds; the R partial sums of the 32 lanes are folded together (lanes
// split the sums between them on the way, 6 fp64 shuffles for 4 sums instead of 20).  Then a warp per query block finds the
// n-th largest key bit by bit and writes the blocks above it, and as many equal to it as there is room for, in order.
// Shared memory: keys [R][total].
template <int D, int R>
__global__ void __launch_bounds__(kSelectThreads)
block_select_kernel(const SelectArgs a, const KeyBlocks kb) {
  static_assert(R == 4 || R == 1, "the fold of the partial sums is written for four sums or one");
  extern __shared__ unsigned long long s_key[];
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int q0 = blockIdx.x * R, h = blockIdx.y, b = blockIdx.z;
  const int rows = min(R, a.q_blocks - q0);
  double q[R][kPer];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      q[r][e] = r < rows ? static_cast<double>(
                               a.q_mean[((static_cast<long long>(b) * a.heads + h) * a.q_blocks + q0 + r) * D + lane * kPer + e])
                         : 0.0;
  const int chunk_blocks = kb.total - kb.ctx, slots = kb.sink_slots + kb.win_slots;
  const float* ctx = a.pooled + static_cast<long long>(a.cache_shared ? 0 : b) * a.heads * slots * kb.per_frame * D +
                     static_cast<long long>(h) * slots * kb.per_frame * D;
  const float* own = a.kc_mean + (static_cast<long long>(b) * a.heads + h) * chunk_blocks * D;
  for (int j = warp; j < kb.total; j += kSelectWarps) {
    const float* src;
    bool keep;
    if (j < kb.ctx) {
      const int f = j / kb.per_frame;
      src = ctx + (static_cast<long long>(key_block_slot(kb, f)) * kb.per_frame + (j - f * kb.per_frame)) * D;
      keep = a.keep_sink && f < kb.sink_held;
    } else {
      src = own + static_cast<long long>(j - kb.ctx) * D;
      keep = a.keep_chunk;
    }
    double k[kPer], s[R];
    if constexpr (kPer == 4) {
      const float4 v = *reinterpret_cast<const float4*>(src + lane * 4);
      k[0] = v.x; k[1] = v.y; k[2] = v.z; k[3] = v.w;
    } else {
      const float2 v = *reinterpret_cast<const float2*>(src + lane * 2);
      k[0] = v.x; k[1] = v.y;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = 0.0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) s[r] = fma(q[r][e], k[e], s[r]);
    }
    double sum;
    int row = 0;
    if constexpr (R == 4) {
      const bool up = lane & 16, left = lane & 8;
      double x = up ? s[2] : s[0], y = up ? s[3] : s[1];
      x += __shfl_xor_sync(0xffffffffu, up ? s[0] : s[2], 16);
      y += __shfl_xor_sync(0xffffffffu, up ? s[1] : s[3], 16);
      sum = left ? y : x;
      sum += __shfl_xor_sync(0xffffffffu, left ? x : y, 8);
      row = (up ? 2 : 0) + (left ? 1 : 0);
    } else {
      sum = s[0];
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    if ((lane & 7) == 0 && (R == 4 || lane == 0))
      s_key[static_cast<long long>(row) * kb.total + j] = keep ? kKeptKey : order_key(sum);
  }
  __syncthreads();
  for (int r = warp; r < rows; r += kSelectWarps) {
    const unsigned long long* key = s_key + static_cast<long long>(r) * kb.total;
    int* out = a.blocks + ((static_cast<long long>(b) * a.heads + h) * a.q_blocks + q0 + r) * a.n_select;
    const int want = min(a.n_select, kb.total);
    unsigned long long cut = 0;   // the want-th largest key: the largest value that at least `want` keys reach
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long cand = cut | (1ull << bit);
      int n = 0;
      for (int j = lane; j < kb.total; j += 32) n += key[j] >= cand;
      if (__reduce_add_sync(0xffffffffu, n) >= want) cut = cand;
    }
    int above = 0;
    for (int j = lane; j < kb.total; j += 32) above += key[j] > cut;
    int ties = want - __reduce_add_sync(0xffffffffu, above);
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
}

}  // namespace astro
