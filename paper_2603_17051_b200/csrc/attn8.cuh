// Attention over a cache held in 8 bits (kv_quant.cuh), the chunk's own keys in bf16:
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - LSE_i),  k_j = 2^ek_j c_j for the cache's rows.
//
// Many queries: the cached rows are turned into bf16 (exactly: kv_quant.cuh) once per call, in the order of the storage, and the
// dense kernels run over them.  Turning them inside the attention kernel would be done again by each of the 37 query tiles of a
// chunk; once costs 3 bytes of traffic per element: 42 us (260 MB, 6.2 TB/s) beside the 635 of 4680 queries over 32760 keys, 12 heads.
//
// Few queries: a kernel of its own that reads the codes and nothing else.  Bandwidth: 2 (D + 1) bytes per key and head: 4 x 12 lists of
// 18720 keys, one query each, in 39 us (232 MB, 5.9 TB/s), and 4 for joining them.
// mma.sync does the products (16 keys x 8 queries x 16 elements; a tcgen05 tile of 128 queries would be 1/16 full, and its
// operands would have to go through shared memory), scores as S^T = K Q^T and O^T = V^T P^T, so that 8 queries fill a tile.
//   The elements of a head are summed in whatever order suits: lane (g, t) of a warp takes 32 consecutive codes of key g from 32 t on
//   for K (16 from 16 t at head_dim 64), and codes 16 g .. 16 g + 15 of keys 2t, 2t+1, 2t+8, 2t+9 for V; Q is brought into the same
//   order, O leaves in it.  P^T changes from its place as a result into that of an operand by movmatrix.
//   The operands are fp16, which holds every e4m3 number: one instruction turns two codes.  A query is multiplied by the power
//   of two that brings its largest element to 2^14 (elements keep all of bf16's bits down to 2^-31 of it, fewer down to 2^-38,
//   and vanish below).
//   2^ek multiplies the score; 2^ev joins the weight: w = exp2(s + ev - M) with M a running maximum of s + ev, rounded to fp16
//   (half a step, 2^-11 of a weight), while the row sum has a reference m of its own and takes fp32 weights.  A step with a weight
//   below 2^-22 of 2^M, of which fp16 would leave less than eight bits or nothing, takes bf16 weights and codes instead (half a
//   step, 2^-8): beside a far larger value row the others may still be all that an element is made of.  What is below 2^-120 of the
//   largest vanishes.  (Call of 4 x 12 lists of 18720 keys, one query each: 44.5 us, 45.2 with scores so far apart that nearly every step is
//   one in bf16; 40 rows over 8001 keys, head_dim 64: 22.7 and 24.7.  Bf16 without a second reference took 8 instructions per pair
//   of pairs of codes and 506 per step: 50 us of kernel in the first case.)
//   A warp streams its own tiles: one lane has 32 rows of K and of V brought by TMA into a ring that no other warp touches,
//   swizzled so that no two lanes of a quarter warp meet in a bank.  (The same bytes by cp.async, 16 per lane, came at 4.8 TB/s
//   whatever the warps did with them.)  References move (all lanes agreeing) when exceeded by more than 8.
//   Over one stored prefix the queries of all samples are the rows of one list.  Warps take 16-key steps of their CTA's range
//   in turn and are joined in shared memory; CTAs that share a list leave normalised parts and their LSE for
//   sparse_combine_kernel.
#pragma once
#include "attn_common.cuh"
#include "kv_quant.cuh"

#include <cfloat>

namespace astro {

// ---------------------------------------------------------------------------------- cached rows into bf16
// grid.x: ((sample, head), piece of its rows), pieces fastest, grid.y: 0: K, 1: V.  The rows of a (sample, head) are one or two
// runs of the storage and become one run of the output [B_c, H, n, D].
struct Expand8 {
  const uint8_t *k, *v, *k_exp, *v_exp;
  __nv_bfloat16 *k_out, *v_out;
  long long slot_tokens;
  int pieces, start0, count0, start1, n;     // logical row r sits at start0 + r, or from count0 on at start1 + r - count0
};
constexpr int kExpandThreads = 256, kExpandRows = 8;

template <int D>
__global__ void __launch_bounds__(kExpandThreads) expand8_kernel(const Expand8 a) {
  constexpr int kLanes = D / 8, kPerPass = kExpandThreads / kLanes;
  const int part = threadIdx.x % kLanes;
  const long long list = blockIdx.x / a.pieces;
  const int r0 = (blockIdx.x - static_cast<int>(list) * a.pieces) * (kPerPass * kExpandRows) + threadIdx.x / kLanes;
  const uint8_t* codes = (blockIdx.y ? a.v : a.k) + list * a.slot_tokens * D + part * 8;
  const uint8_t* exps = (blockIdx.y ? a.v_exp : a.k_exp) + list * a.slot_tokens;
  __nv_bfloat16* out = (blockIdx.y ? a.v_out : a.k_out) + list * a.n * D + part * 8;
  uint2 w[kExpandRows];
  uint32_t e[kExpandRows];
#pragma unroll
  for (int i = 0; i < kExpandRows; ++i) {
    const int r = r0 + i * kPerPass;
    if (r >= a.n) continue;
    const long long row = r < a.count0 ? a.start0 + r : a.start1 + (r - a.count0);
    w[i] = __ldcs(reinterpret_cast<const uint2*>(codes + row * D));
    e[i] = exps[row];
  }
#pragma unroll
  for (int i = 0; i < kExpandRows; ++i) {
    const int r = r0 + i * kPerPass;
    if (r >= a.n) continue;
    const float s = exp_byte_to_float(e[i]);
    const float2 p[4] = {e4m3_to_floats(w[i].x), e4m3_to_floats(w[i].x >> 16), e4m3_to_floats(w[i].y), e4m3_to_floats(w[i].y >> 16)};
    const float f[8] = {p[0].x * s, p[0].y * s, p[1].x * s, p[1].y * s, p[2].x * s, p[2].y * s, p[3].x * s, p[3].y * s};
    store8(out + static_cast<long long>(r) * D, f);
  }
}

// delta from the weights, sum_j p_ij dO_i . v_j, instead of dO_i . O_i with the rounded O, over few keys (here, a warp per (sample,
// head, query) of the expanded rows kx, vx) and for few queries (kDqDelta): where one key has nearly all the weight of a row, dS is far
// smaller than delta, and half a step of O's, 2^-8 of delta, is per cents of it (3 queries over 325 keys of uneven sizes: dQ 5.5e-3
// off with the rounded O, 2.6e-3 from the weights).  Among many rows those with large gradients outweigh such a one.
constexpr int kFewRows = 8;
constexpr int kShortKeys = 64;
struct ShortDelta8 {
  const __nv_bfloat16 *q, *d_o, *kx, *vx, *kc, *vc;
  const float* lse;
  float* delta;
  long long rows;
  int heads, n_q, n_ctx, n_kc, shared;
  float scale_log2;
};
template <int D>
__global__ void __launch_bounds__(128) attn8_short_delta_kernel(const ShortDelta8 a) {
  constexpr int kPer = D / 32;
  const long long at = blockIdx.x * 4ll + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (at >= a.rows) return;
  const long long bh = at / a.n_q, b = bh / a.heads;
  const int i = static_cast<int>(at - bh * a.n_q), h = static_cast<int>(bh - b * a.heads);
  const long long row = ((b * a.n_q + i) * a.heads + h) * D + lane * kPer;
  float q[kPer], g[kPer], sum = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    q[e] = __bfloat162float(a.q[row + e]);
    g[e] = __bfloat162float(a.d_o[row + e]);
  }
  const float lse2 = a.lse[at] * 1.4426950408889634f;
  for (int j = 0; j < a.n_ctx + a.n_kc; ++j) {
    const bool ctx = j < a.n_ctx;
    const long long from = ctx ? (((a.shared ? 0 : b) * a.heads + h) * a.n_ctx + j) * D + lane * kPer
                               : ((b * a.n_kc + (j - a.n_ctx)) * a.heads + h) * D + lane * kPer;
    float s = 0.f, dp = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      s = fmaf(q[e], __bfloat162float((ctx ? a.kx : a.kc)[from + e]), s);
      dp = fmaf(g[e], __bfloat162float((ctx ? a.vx : a.vc)[from + e]), dp);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      s += __shfl_xor_sync(0xffffffffu, s, d);
      dp += __shfl_xor_sync(0xffffffffu, dp, d);
    }
    sum = fmaf(fast_exp2(s * a.scale_log2 - lse2), dp, sum);
  }
  if (lane == 0) a.delta[at] = sum;
}

// A softmax over one key is constant: no gradient for its queries and for it, where the kernels leave fp32's rounding of
// dP - delta.  What is NaN or infinite stays.  n pairs of elements.
__global__ void __launch_bounds__(256) attn8_one_key_kernel(__nv_bfloat162* x, long long n) {
  const long long i = blockIdx.x * 256ll + threadIdx.x;
  if (i >= n) return;
  const float2 v = __bfloat1622float2(x[i]);
  x[i] = __floats2bfloat162_rn(fabsf(v.x) < INFINITY ? 0.f : v.x, fabsf(v.y) < INFINITY ? 0.f : v.y);
}

// dQ from its parts (DqParts), in their order: four elements a thread.
template <int D>
__global__ void __launch_bounds__(256) attn8_join_dq_kernel(const float* parts, int splits, long long rows, int n_q, int heads, float scale,
                                                            __nv_bfloat16* dq) {
  dependency_wait();
  const long long at = blockIdx.x * 256ll + threadIdx.x, row = at / (D / 4);
  if (row >= rows) return;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int p = 0; p < splits; ++p) {
    const float4 v = reinterpret_cast<const float4*>(parts)[p * rows * (D / 4) + at];
    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
  }
  const long long bh = row / n_q, b = bh / heads;
  const long long to = ((b * n_q + (row - bh * n_q)) * heads + (bh - b * heads)) * D + at % (D / 4) * 4;
  *reinterpret_cast<uint2*>(dq + to) = make_uint2(pack_bf16(sum.x * scale, sum.y * scale), pack_bf16(sum.z * scale, sum.w * scale));
}

// ---------------------------------------------------------------------------------- few queries
constexpr int kFewStep = 32;                       // keys of a step: two tiles of 16, whose latencies overlap

// 8 * NT queries per CTA; at head_dim 128 twice the queries leave registers for fewer warps (at 64 twelve warps with four stages
// each take 85 us for 128 queries of 12 heads over 28080 keys; before the look at the weights' range 81, and eight with five 92).
template <int D, int NT> struct FewShape {
  static constexpr int kWarps = NT == 1 || D == 64 ? 12 : 8, kThreads = 32 * kWarps;
  static constexpr int kPieces = D / 64;           // 16-byte pieces of a key's K per lane
  static constexpr int kVBytes = D / 8;            // bytes of a key's V per lane: 16 or 8
  static constexpr int kStageBytes = 2 * kFewStep * D;   // K, then V
  static constexpr int kStages = D == 128 ? 1 + NT : 4;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  static constexpr int kJoined = kWarps * 8 * NT * (D + 4) * 4;               // the warps' outputs and statistics, behind the loop
  static constexpr int kBars = kRing > kJoined ? kRing : kJoined;
  static constexpr int kTotal = kBars + kWarps * kStages * 8 + 16 + 1024;
};

struct FewArgs {
  const __nv_bfloat16 *q, *kc, *vc;
  const uint8_t *k_exp, *v_exp;
  __nv_bfloat16* o;
  float* lse;              // may be null
  float *part_o, *part_lse;  // when splits > 1
  long long slot_tokens;
  int start0, count0, start1, count1, n_kc;   // the held rows' two runs in the storage
  int batch, heads, n_q, splits;
  int rows;                // of a list: n_q, or batch * n_q over one prefix
  int shared;              // 1: one prefix for all samples
  float scale_log2;
};

struct FewMaps {
  CUtensorMap k[2], v[2];   // {code, token up to the run's end, list} of both runs
};
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tmap, uint64_t* bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// Byte offset of 16-byte chunk `chunk` of row `row` in a tile of rows of D bytes, as TMA's swizzle over D bytes leaves it.
template <int D> __device__ __forceinline__ int swizzled(int row, int chunk) {
  return row * D + ((chunk ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4);
}

// Transposes an 8 x 8 matrix of 16-bit elements, a row per quad of lanes, two neighbours per lane.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

constexpr float kFewSlack = 8.f, kFewBias = 6.f, kFewUnit = 1.f / 64.f;   // weights reach 2^14 at most; 2^-kFewBias
constexpr float kFewRange = 22.f;                  // in fp16 weights from 2^(kFewBias - 22) on are at most 2^-9 of themselves off

// The running state of a warp: 8 * NT queries.  O is held in units of 2^(top - kFewBias).
template <int D, int NT> struct FewState {
  float o[NT][D / 16][4];   // rows (elements) g and g + 8 of tile j = elements (D/8) g + 2 j and the next; columns: queries 2t, 2t+1
  float m[NT][2], l[NT][2]; // of queries 2t, 2t+1: reference of the row sum, sum of the lane's own keys
  float top[NT][2];         // reference of the weights times their values' factors
  __device__ void clear() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = top[n][0] = top[n][1] = -FLT_MAX;   // below every score; differences to it are no NaN
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
    }
  }
  // Scores of keys g (s[..][..][0..1]) and g + 8 (s[..][..][2..3]) of TILES tiles in log2 units, -infinity where there is no key,
  // and the exponents of their values -> the weights as the operands of O^T = V^T P^T, in bf16 where it returns true (kBf16: always).
  template <bool kBf16, int TILES>
  __device__ __forceinline__ bool weigh(const float (&s)[TILES][NT][4], const float (&e)[TILES][2], uint32_t (&b)[TILES][NT][2]) {
    bool over = false, small = false, wide = kBf16;
    float least[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = -INFINITY, y = -INFINITY;
        least[n][c] = INFINITY;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          x = max3(x, s[i][n][c], s[i][n][c + 2]);
          y = max3(y, s[i][n][c] + e[i][0], s[i][n][c + 2] + e[i][1]);
          least[n][c] = min3(least[n][c], s[i][n][c] + e[i][0], s[i][n][c + 2] + e[i][1]);
        }
        over = over || x > m[n][c] + kFewSlack || y > top[n][c] + kFewSlack;
        small = small || (!kBf16 && least[n][c] < top[n][c] - kFewRange);
      }
    if (__any_sync(0xffffffffu, over || small)) {   // rare, or there are places without a key
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = m[n][c], y = top[n][c];
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
              x = max3(x, s[i][n][c], s[i][n][c + 2]);
              y = max3(y, s[i][n][c] + e[i][0], s[i][n][c + 2] + e[i][1]);
            }
#pragma unroll
            for (int d = 4; d < 32; d *= 2) {
              x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
              y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, d));
            }
            l[n][c] *= fast_exp2(m[n][c] - x);
            const float alpha = fast_exp2(top[n][c] - y);
            m[n][c] = x;
            top[n][c] = y;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
              o[n][j][c] *= alpha;
              o[n][j][c + 2] *= alpha;
            }
          }
      }
      if constexpr (!kBf16) {
        small = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) small = small || least[n][0] < top[n][0] - kFewRange || least[n][1] < top[n][1] - kFewRange;
        if (__any_sync(0xffffffffu, small)) {
          small = false;
#pragma unroll
          for (int i = 0; i < TILES; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < 4; ++x) small = small || (s[i][n][x] != -INFINITY && s[i][n][x] + e[i][x / 2] < top[n][x % 2] - kFewRange);
          wide = __any_sync(0xffffffffu, small);
        }
      }
    }
    auto weights = [&](auto is_wide) {
      constexpr bool kWide = decltype(is_wide)::value;
#pragma unroll
      for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float w[4];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float wref = top[n][c] - kFewBias;
            l[n][c] += fast_exp2(s[i][n][c] - m[n][c]) + fast_exp2(s[i][n][c + 2] - m[n][c]);
            w[c] = fast_exp2(s[i][n][c] + (e[i][0] - wref));
            w[c + 2] = fast_exp2(s[i][n][c + 2] + (e[i][1] - wref));
          }
          b[i][n][0] = transpose_8x8(kWide ? pack_bf16(w[0], w[1]) : pack_half(w[0], w[1]));
          b[i][n][1] = transpose_8x8(kWide ? pack_bf16(w[2], w[3]) : pack_half(w[2], w[3]));
        }
    };
    if (kBf16 || wide) weights(std::true_type{});
    else weights(std::false_type{});
    return wide;
  }
};

// grid.x: (tile of 8 NT rows, split) with the split fastest, grid.y: head, grid.z: sample (one over a shared prefix).
template <int D, int NT>
__global__ void __launch_bounds__(FewShape<D, NT>::kThreads, 1) attn8_few_kernel(const __grid_constant__ FewMaps maps, const __grid_constant__ FewArgs a) {
  using S = FewShape<D, NT>;
  constexpr int kFewWarps = S::kWarps, kFewThreads = S::kThreads;
  extern __shared__ uint8_t few_smem_raw[];
  uint8_t* few_smem = align_1024(few_smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % a.splits, row0 = blockIdx.x / a.splits * (8 * NT);
  const int h = blockIdx.y, bz = blockIdx.z;
  const long long list = static_cast<long long>(bz) * a.heads + h;
  const uint8_t *ke = a.k_exp + list * a.slot_tokens, *ve = a.v_exp + list * a.slot_tokens;
  uint8_t* ring = few_smem + warp * (S::kStages * S::kStageBytes);
  uint64_t* full = reinterpret_cast<uint64_t*>(few_smem + S::kBars) + warp * S::kStages;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(few_smem + S::kBars + kFewWarps * S::kStages * 8);
  if (lane == 0) {
    for (int i = 0; i < S::kStages; ++i) mbar_init(full + i, 1);
    fence_mbar_init();
  }
  if (threadIdx.x == 0) *abort_flag = 0;
  dependents_may_start();   // the joining kernel waits for the whole grid where it begins
  __syncthreads();
  // row of the list -> sample and query
  auto sample_of = [&](int row) { return a.shared ? row / a.n_q : bz; };
  auto query_of = [&](int row) { return a.shared ? row % a.n_q : row; };

  // this CTA's steps: those of the cache first, then those of the chunks of the samples that the rows belong to
  const int row_end = min(row0 + 8 * NT, a.rows), first_sample = sample_of(row0);
  const int steps0 = (a.count0 + kFewStep - 1) / kFewStep, ctx_steps = steps0 + (a.count1 + kFewStep - 1) / kFewStep;
  const int chunk_steps = (a.n_kc + 15) / 16;   // the chunk's: one tile
  const int steps = ctx_steps + (sample_of(row_end - 1) - first_sample + 1) * chunk_steps;
  const int each = steps / a.splits, rest = steps % a.splits;
  const int first = split * each + min(split, rest), last = first + each + (split < rest ? 1 : 0);
  const int ctx_last = min(last, ctx_steps);

  // the first row of a step in the storage, and how many of its 32 are there
  auto row_of_step = [&](int step) { return step < steps0 ? a.start0 + step * kFewStep : a.start1 + (step - steps0) * kFewStep; };
  auto rows_left = [&](int step) { return step < steps0 ? a.count0 - step * kFewStep : a.count1 - (step - steps0) * kFewStep; };
  // Rows behind a run's end come as zeros.  All lanes have read the stage before.
  auto fetch = [&](int step, int stage) {
    __syncwarp();
    if (lane == 0 && step < ctx_last) {
      const int run = step < steps0 ? 0 : 1, row = row_of_step(step);
      const uint32_t dst = smem_u32(ring + stage * S::kStageBytes);
      mbar_arrive_expect_tx(full + stage, S::kStageBytes);
      tma_load_3d(dst, &maps.k[run], full + stage, 0, row, static_cast<int>(list));
      tma_load_3d(dst + kFewStep * D, &maps.v[run], full + stage, 0, row, static_cast<int>(list));
    }
  };
  uint32_t k_next[2][2], v_next[2][2];   // exponent bytes of keys g, g + 8 of both tiles
  auto fetch_exps = [&](int step) {
    if (step < ctx_last) {
      const int row = row_of_step(step), most = rows_left(step) - 1;
#pragma unroll
      for (int tile = 0; tile < 2; ++tile)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = row + min(16 * tile + g + 8 * i, most);
          k_next[tile][i] = ke[r];
          v_next[tile][i] = ve[r];
        }
    }
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) fetch(first + warp + i * kFewWarps, i);
  fetch_exps(first + warp);

  // Q in the order of the K pieces: elements 16 (kPieces t + c) + 4 x + {0, 1} and {2, 3} of query 8 n + g
  uint32_t qf[NT][S::kPieces][4][2];
  auto load_q = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = min(row0 + 8 * n + g, row_end - 1);
      const uint4* src = reinterpret_cast<const uint4*>(a.q + ((static_cast<long long>(sample_of(row)) * a.n_q + query_of(row)) * a.heads + h) * D);
#pragma unroll
      for (int c = 0; c < S::kPieces; ++c)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint4 w = src[2 * (S::kPieces * t + c) + x];
          qf[n][c][2 * x][0] = w.x; qf[n][c][2 * x][1] = w.y;
          qf[n][c][2 * x + 1][0] = w.z; qf[n][c][2 * x + 1][1] = w.w;
        }
    }
  };
  load_q();
  float unit[NT][2];    // of queries 2t, 2t+1: what turns a sum of products into a score in log2 units, without the key's factor
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    uint32_t big = 0;   // the largest finite magnitude's bits
#pragma unroll
    for (int x = 0; x < S::kPieces * 8; ++x) {
      const uint32_t w = qf[n][x / 8][x / 2 % 4][x % 2], lo = w << 16 & 0x7fffffffu, hi = w & 0x7fff0000u;
      big = max(big, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
    }
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    const int up = min(14 - (static_cast<int>(big >> 23) - 127), 120);   // -113 at least
    const float factor = __uint_as_float(static_cast<uint32_t>(127 + up) << 23);
    const float back = __uint_as_float(static_cast<uint32_t>(127 - up) << 23) * a.scale_log2;
#pragma unroll
    for (int x = 0; x < S::kPieces * 8; ++x) {
      uint32_t& w = qf[n][x / 8][x / 2 % 4][x % 2];
      w = pack_half(__uint_as_float(w << 16) * factor, __uint_as_float(w & 0xffff0000u) * factor);
    }
    unit[n][0] = __shfl_sync(0xffffffffu, back, 8 * t);
    unit[n][1] = __shfl_sync(0xffffffffu, back, 8 * t + 4);
  }
  FewState<D, NT> st;
  st.clear();

  int stage = 0, round = 0;
  for (int step = first + warp; step < ctx_last; step += kFewWarps) {
    // into the stage that the step before has been read out of
    fetch(step + (S::kStages - 1) * kFewWarps, stage == 0 ? S::kStages - 1 : stage - 1);
    if (!mbar_wait_ok(full + stage, round & 1, abort_flag)) break;
    const uint8_t* held = ring + stage * S::kStageBytes;
    float ks[2][2], ve_log2[2][2];
#pragma unroll
    for (int tile = 0; tile < 2; ++tile)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ks[tile][i] = exp_byte_to_float(k_next[tile][i]);
        ve_log2[tile][i] = static_cast<float>(static_cast<int>(v_next[tile][i]) - 127);
      }
    fetch_exps(step + kFewWarps);
    float s[2][NT][4];
#pragma unroll
    for (int tile = 0; tile < 2; ++tile)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[tile][n][e] = 0.f;
#pragma unroll
    for (int c = 0; c < S::kPieces; ++c)
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const uint4 x = *reinterpret_cast<const uint4*>(held + swizzled<D>(16 * tile + g, S::kPieces * t + c));
        const uint4 y = *reinterpret_cast<const uint4*>(held + swizzled<D>(16 * tile + g + 8, S::kPieces * t + c));
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a0 = e4m3_to_half2(xw[i]), a2 = e4m3_to_half2(xw[i] >> 16);
          const uint32_t a1 = e4m3_to_half2(yw[i]), a3 = e4m3_to_half2(yw[i] >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_16x8x16<false>(s[tile][n], a0, a1, a2, a3, qf[n][c][i][0], qf[n][c][i][1]);
        }
      }
#pragma unroll
    for (int tile = 0; tile < 2; ++tile)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[tile][n][e] *= ks[tile][e / 2] * unit[n][e % 2];
    const int left = rows_left(step);
    if (left < kFewStep) {
#pragma unroll
      for (int tile = 0; tile < 2; ++tile)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * tile + g + 8 * (e / 2) >= left) s[tile][n][e] = -INFINITY;
    }
    uint32_t p[2][NT][2];
    const bool wide = st.template weigh<false, 2>(s, ve_log2, p);
    auto add_values = [&](auto is_wide) {
      constexpr bool kWide = decltype(is_wide)::value;
      auto operand = [](uint32_t codes) {
        if constexpr (!kWide) return e4m3_to_half2(codes);
        else {
          const float2 f = e4m3_to_floats(codes);
          return pack_bf16(f.x, f.y);
        }
      };
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        // V: words of keys 2t, 2t+1, 2t+8, 2t+9
        uint32_t w[4][S::kVBytes / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 16 * tile + 2 * t + (i & 1) + 8 * (i >> 1);
          if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(held + kFewStep * D + swizzled<D>(r, g));
            w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(held + kFewStep * D + swizzled<D>(r, g >> 1) + 8 * (g & 1));
            w[i][0] = x.x; w[i][1] = x.y;
          }
        }
#pragma unroll
        for (int i = 0; i < S::kVBytes / 4; ++i)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t sel = half ? 0x7362u : 0x5140u;   // codes of two elements, keys side by side
            const uint32_t x = __byte_perm(w[0][i], w[1][i], sel), y = __byte_perm(w[2][i], w[3][i], sel);
            const uint32_t a0 = operand(x), a1 = operand(x >> 16), a2 = operand(y), a3 = operand(y >> 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_16x8x16<kWide>(st.o[n][2 * i + half], a0, a1, a2, a3, p[tile][n][0], p[tile][n][1]);
          }
      }
    };
    if (wide) add_values(std::true_type{});
    else add_values(std::false_type{});
    if (++stage == S::kStages) { stage = 0; ++round; }
  }

  // the chunks' own keys, bf16 [B, n_kc, H, D]; the warps take them in the order in which the cache's steps would have gone on
  int step = first + warp;
  if (step < ctx_steps) step += (ctx_steps - step + kFewWarps - 1) / kFewWarps * kFewWarps;
  if (step < last) load_q();
  for (; step < last; step += kFewWarps) {
    const int b = first_sample + (step - ctx_steps) / chunk_steps, key0 = (step - ctx_steps) % chunk_steps * 16;
    auto row_of = [&](const __nv_bfloat16* base, int key) {
      return base + ((static_cast<long long>(b) * a.n_kc + min(key, a.n_kc - 1)) * a.heads + h) * D;
    };
    float s[1][NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[0][n][e] = 0.f;
    const uint4 *k0 = reinterpret_cast<const uint4*>(row_of(a.kc, key0 + g)), *k1 = reinterpret_cast<const uint4*>(row_of(a.kc, key0 + g + 8));
#pragma unroll
    for (int c = 0; c < S::kPieces; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 x = k0[2 * (S::kPieces * t + c) + i], y = k1[2 * (S::kPieces * t + c) + i];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_16x8x16<true>(s[0][n], x.x, y.x, x.y, y.y, qf[n][c][2 * i][0], qf[n][c][2 * i][1]);
          mma_16x8x16<true>(s[0][n], x.z, y.z, x.w, y.w, qf[n][c][2 * i + 1][0], qf[n][c][2 * i + 1][1]);
        }
      }
    const int left = a.n_kc - key0;
    // a sample's keys are seen by its own queries
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[0][n][e] = g + 8 * (e / 2) < left && sample_of(row0 + 8 * n + 2 * t + e % 2) == b ? s[0][n][e] * a.scale_log2 : -INFINITY;
    // no weight for those who do not see the key, whatever its value holds: 0 * NaN would reach them
    uint32_t p[1][NT][2];
    const float none[1][2] = {{0.f, 0.f}};
    st.template weigh<true, 1>(s, none, p);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {       // 8 elements of the lane's D/8
      uint32_t w[4][4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint4 x = reinterpret_cast<const uint4*>(row_of(a.vc, key0 + 2 * t + (r & 1) + 8 * (r >> 1)) + g * (D / 8))[i];
        w[r][0] = x.x; w[r][1] = x.y; w[r][2] = x.z; w[r][3] = x.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float add[4] = {0.f, 0.f, 0.f, 0.f};
          mma_16x8x16<true>(add, __byte_perm(w[0][j], w[1][j], 0x5410), __byte_perm(w[0][j], w[1][j], 0x7632),
                            __byte_perm(w[2][j], w[3][j], 0x5410), __byte_perm(w[2][j], w[3][j], 0x7632), p[0][n][0], p[0][n][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (sample_of(row0 + 8 * n + 2 * t + e % 2) == b) st.o[n][4 * i + j][e] += add[e];
        }
    }
  }

  // ---- the warps' outputs joined: [warp][query][D], then [warp][query] of references and sums
  settle_after_abort(abort_flag);
  __syncthreads();
  float* out = reinterpret_cast<float*>(few_smem);
  float4* stats = reinterpret_cast<float4*>(out + kFewWarps * 8 * NT * D);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float l = st.l[n][c];
#pragma unroll
      for (int x = 4; x < 32; x *= 2) l += __shfl_xor_sync(0xffffffffu, l, x);
      const int i = warp * 8 * NT + 8 * n + 2 * t + c;
      if (g == 0) stats[i] = make_float4(st.m[n][c], l, st.top[n][c], 0.f);
      float* dst = out + i * D + g * (D / 8);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) *reinterpret_cast<float2*>(dst + 2 * j) = make_float2(st.o[n][j][c], st.o[n][j][c + 2]);
    }
  __syncthreads();
  constexpr int kVecs = 8 * NT * D / 2;
  for (int x = threadIdx.x; x < kVecs; x += kFewThreads) {
    const int i = x / (D / 2), d = x % (D / 2) * 2, row = row0 + i;
    if (row >= a.rows) continue;
    float ref = -FLT_MAX;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) ref = fmaxf(ref, stats[w * 8 * NT + i].x);
    float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float4 f = stats[w * 8 * NT + i];
      const float2 v = *reinterpret_cast<const float2*>(out + (w * 8 * NT + i) * D + d);
      // by halves: 2^(f.z - ref) alone is no float where all values are of the smallest rows.  0 for a warp without keys, here and next
      const float half = fast_exp2(0.5f * (f.z - ref));
      l = fmaf(fast_exp2(f.x - ref), f.y, l);
      o0 = fmaf(half, v.x * kFewUnit * half, o0);
      o1 = fmaf(half, v.y * kFewUnit * half, o1);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float lse = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.6931471805599453f;
    const int b = sample_of(row), q = query_of(row);
    const long long at = (static_cast<long long>(b) * a.heads + h) * a.n_q + q;
    if (a.splits > 1) {
      const long long rows = static_cast<long long>(a.batch) * a.heads * a.n_q;
      *reinterpret_cast<float2*>(a.part_o + (split * rows + at) * D + d) = make_float2(o0 * inv, o1 * inv);
      if (d == 0) a.part_lse[split * rows + at] = lse;
    } else {
      *reinterpret_cast<uint32_t*>(a.o + ((static_cast<long long>(b) * a.n_q + q) * a.heads + h) * D + d) = pack_bf16(o0 * inv, o1 * inv);
      if (d == 0 && a.lse != nullptr) a.lse[at] = lse;
    }
  }
}
}  // namespace astro
