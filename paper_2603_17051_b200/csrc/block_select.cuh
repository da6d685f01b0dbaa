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

// Sums of bf16 values in fp64 without a conversion per value (those run at a quarter of the adds' rate or less): the bits of a
// bf16, moved to the places of an fp64's sign, exponent and mantissa, are that value times 2^-896, zeros and denormal
// values included; the sum is scaled back once.  Infinities and NaN have no such image (`seen` collects the magnitudes so
// that they are noticed).
__device__ __forceinline__ void add_scaled(double& lo, double& hi, uint32_t pair) {
  lo += __hiloint2double(static_cast<int>(((pair << 13) & 0x0fffe000u) | ((pair << 16) & 0x80000000u)), 0);
  hi += __hiloint2double(static_cast<int>(((pair >> 3) & 0x0fffe000u) | (pair & 0x80000000u)), 0);
}

// One block of tokens of one head per thread block: D/8 threads side by side hold 8 elements each, the others walk the
// tokens, all of a thread's loads in flight at once; partial sums meet in shared memory.  Bandwidth bound.
// grid.x = blocks of source 0, then of source 1 (n0 of the first); grid.y = head, grid.z = sample.  cache_source: source 0 is
// the cache storage, and grid.x walks the blocks of the frames from logical frame `frame0` on.
template <int D>
__global__ void __launch_bounds__(kPoolThreads)
block_pool_kernel(const PoolSource s0, const PoolSource s1, const int n0, const KeyBlocks kb, const int frame0,
                  const int cache_source) {
  constexpr int kCols = D / 8, kRows = kPoolThreads / kCols, kDeep = kTile / kRows;   // a block has at most kTile tokens
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
  uint4 v[kDeep];
#pragma unroll
  for (int u = 0; u < kDeep; ++u) {
    const int t = row + u * kRows;
    v[u] = t < count ? *reinterpret_cast<const uint4*>(src + t * s.st) : make_uint4(0, 0, 0, 0);
  }
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0;
  uint32_t seen = 0;
#pragma unroll
  for (int u = 0; u < kDeep; ++u) {
    const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      add_scaled(acc[2 * e], acc[2 * e + 1], w[e]);
      seen = __vmaxu2(seen, w[e] & 0x7fff7fffu);
    }
  }
  double unscale = ldexp(1.0, 896);
  if ((seen & 0xffffu) >= 0x7f80u || (seen >> 16) >= 0x7f80u) {   // again with true conversions; scaled down, see below
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0;
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
      const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = __bfloat1622float2(p[e]);
        acc[2 * e] += static_cast<double>(f.x);
        acc[2 * e + 1] += static_cast<double>(f.y);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= 1.0 / unscale;   // back into the others' scale; a power of two loses nothing
  }
  __shared__ double part[kRows][8][kCols];
#pragma unroll
  for (int e = 0; e < 8; ++e) part[row][e][col] = acc[e];
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kPoolThreads) {
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) sum += part[r][e % 8][e / 8];
    s.out[((b * s.out_b + h * s.out_h) + out_row) * D + e] = static_cast<float>(sum * unscale / static_cast<double>(count));
  }
}

// ------------------------------------------------------------------------------------------------ choice
constexpr int kSelectThreads = 512;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kSelectRows = 8;     // query blocks of one MMA tile

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

// Up to eight query blocks of one head per thread block.  Scores: a warp per eight key blocks, fp64 MMAs over the head
// dimension; the contraction index is dealt to the lanes so that each reads 16 contiguous bytes of a row (the same
// order on both sides, so nothing else changes).  Then a warp per query block finds the n-th largest key bit by bit, stopping
// as soon as a candidate separates exactly n, and writes the blocks above it, and as many equal to it as there is room
// for, in order.  Scores by fused multiply-adds and shuffles, a warp per key block: 42 us for a chunk of 37 x 12 query blocks
// and 273 key blocks against XXX.
// Shared memory: keys [rows][total].
template <int D>
__global__ void __launch_bounds__(kSelectThreads)
block_select_kernel(const SelectArgs a, const KeyBlocks kb) {
  extern __shared__ unsigned long long s_key[];
  constexpr int kSteps = D / 16;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int q0 = blockIdx.x * a.rows, h = blockIdx.y, b = blockIdx.z;
  const int rows = min(a.rows, a.q_blocks - q0);
  const int slots = kb.sink_slots + kb.win_slots, chunk_blocks = kb.total - kb.ctx;
  const float* ctx = a.pooled + static_cast<long long>(a.cache_shared ? 0 : b) * a.heads * slots * kb.per_frame * D +
                     static_cast<long long>(h) * slots * kb.per_frame * D;
  const float* own = a.kc_mean + (static_cast<long long>(b) * a.heads + h) * chunk_blocks * D;
  const int pair = lane >> 2, col = (lane & 3) * 4;
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
    // the want-th largest key: the largest value that at least `want` keys reach; or any value that exactly `want` reach
    unsigned long long cut = 0;
    int reach = kb.total;
    for (int bit = 63; bit >= 0 && reach != want; --bit) {
      const unsigned long long cand = cut | (1ull << bit);
      int n = 0;
      for (int j = lane; j < kb.total; j += 32) n += key[j] >= cand;
      n = __reduce_add_sync(0xffffffffu, n);
      if (n >= want) {
        cut = cand;
        reach = n;
      }
    }
    int above = 0;   // keys over the cut; the rest of the places go to those equal to it, the lower blocks first
    for (int j = lane; j < kb.total; j += 32) above += key[j] > cut;
    int ties = want - __reduce_add_sync(0xffffffffu, above);
    if (reach == want) ties = kb.total;
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
