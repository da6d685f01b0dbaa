// Attention over a cache held in 8 bits (kv_quant.cuh), the chunk's own keys in bf16:
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - LSE_i),  k_j = 2^ek_j c_j for the cache's rows.
//
// Many queries: the cached rows are turned into bf16 (exactly: kv_quant.cuh) once per call, in the order of the frames, and the
// dense kernels run over them.  Turning them inside the attention kernel would be done again by each of the 37 query tiles of a
// chunk; once costs 3 bytes of traffic per element, 40 to 50 us beside the layer's 660.
//
// Few queries: a kernel of its own that reads the codes and nothing else.  Bandwidth: 2 (D + 1) bytes per key and head.
// mma.sync does the products (16 keys x 8 queries x 16 elements; a tcgen05 tile of 128 queries would be 1/16 full, and its
// operands would have to go through shared memory), scores as S^T = K Q^T and O^T = V^T P^T, so that 8 queries fill a tile.
//   The elements of a head are summed in whatever order suits: lane (g, t) of a warp takes 16 consecutive codes of key g at
//   16 t and 64 + 16 t for K, and codes 16 g .. 16 g + 15 of keys 2t, 2t+1, 2t+8, 2t+9 for V, each one 16-byte access; Q is
//   brought into the same order, O leaves in it.  P^T changes from its place as a result into that of an operand by movmatrix.
//   The operands are fp16, which holds every e4m3 number: one instruction turns two codes.  A query is multiplied by the power
//   of two that brings its largest element to 2^14 (elements below 2^-38 of it vanish, the others keep all of bf16's bits).
//   2^ek multiplies the score; 2^ev joins the weight: w = exp2(s + ev - M) with M a running maximum of s + ev, rounded to fp16
//   (half a step, 2^-11 of a weight; those below 2^-31 of the largest vanish), while the row sum has a reference m of its own
//   and takes fp32 weights.  (In bf16, whose range needs no second reference, turning the codes took 8 instructions per pair of
//   pairs and the whole 506 per step: 50 us for 4 x 12 lists of 18720 keys, against 36 of bytes.)
//   Every lane fetches its own 16-byte pieces with cp.async into slots that no other lane touches: a deep ring without a
//   barrier, read back without a bank conflict.  References move (all lanes agreeing) when exceeded by more than 8.
//   Over one stored prefix the queries of all samples are the rows of one list.  Warps take 16-key steps of their CTA's range
//   in turn and are joined in shared memory; CTAs that share a list leave normalised parts and their LSE for
//   sparse_combine_kernel.
#pragma once
#include "attn_common.cuh"
#include "kv_quant.cuh"

namespace astro {

// ---------------------------------------------------------------------------------- cached rows into bf16
// grid.x: pieces of kQuantTokens * rows-per-block tokens, grid.y: (sample, head), grid.z: 0: K, 1: V.  The rows of a (sample,
// head) are one or two runs of the storage and become one run of the output [B_c, H, n, D].
struct Expand8 {
  const uint8_t *k, *v, *k_exp, *v_exp;
  __nv_bfloat16 *k_out, *v_out;
  long long slot_tokens;
  int start0, count0, start1, n;     // logical row r sits at start0 + r, or from count0 on at start1 + r - count0
};
constexpr int kExpandThreads = 256, kExpandRows = 8;

template <int D>
__global__ void __launch_bounds__(kExpandThreads) expand8_kernel(const Expand8 a) {
  constexpr int kLanes = D / 8, kPerPass = kExpandThreads / kLanes;
  dependents_may_start();
  const int part = threadIdx.x % kLanes;
  const int r0 = blockIdx.x * (kPerPass * kExpandRows) + threadIdx.x / kLanes;
  const uint8_t* codes = (blockIdx.z ? a.v : a.k) + static_cast<long long>(blockIdx.y) * a.slot_tokens * D + part * 8;
  const uint8_t* exps = (blockIdx.z ? a.v_exp : a.k_exp) + static_cast<long long>(blockIdx.y) * a.slot_tokens;
  __nv_bfloat16* out = (blockIdx.z ? a.v_out : a.k_out) + static_cast<long long>(blockIdx.y) * a.n * D + part * 8;
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

// ---------------------------------------------------------------------------------- few queries
constexpr int kFewStep = 16;                       // keys of a step

// 8 * NT queries per CTA; twice the queries take twice the registers and half the warps.
template <int D, int NT> struct FewShape {
  static constexpr int kWarps = 16 / NT, kThreads = 32 * kWarps;
  static constexpr int kPieces = D / 64;           // 16-byte pieces of a key's K per lane
  static constexpr int kSlots = 2 * kPieces + 4;   // accesses per lane and step: K of two keys, V of four
  static constexpr int kVBytes = D / 8;            // bytes of a key's V per lane: 16 or 8
  static constexpr int kStageBytes = 32 * (2 * kPieces * 16 + 4 * kVBytes);
  static constexpr int kStages = (D == 128 ? 3 : 6) * NT;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
};

struct FewArgs {
  const __nv_bfloat16 *q, *kc, *vc;
  const uint8_t *k, *v, *k_exp, *v_exp;
  __nv_bfloat16* o;
  float* lse;              // may be null
  float *part_o, *part_lse;  // when splits > 1
  long long slot_tokens;
  int start0, count0, start1, n_ctx, n_kc;
  int batch, heads, n_q, splits;
  int rows;                // of a list: n_q, or batch * n_q over one prefix
  int shared;              // 1: one prefix for all samples
  float scale_log2;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// c[16 x 8] += a[16 x 16] b[16 x 8], bf16 or fp16 products, fp32 sums.
template <bool kBf16>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
  if constexpr (kBf16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

constexpr float kFewSlack = 8.f, kFewBias = 6.f;   // weights reach 2^14 at most

// The running state of a warp: 8 * NT queries.  O is held in units of 2^(top - kFewBias).
template <int D, int NT> struct FewState {
  float o[NT][D / 16][4];   // rows (elements) g and g + 8 of tile j = elements (D/8) g + 2 j and the next; columns: queries 2t, 2t+1
  float m[NT][2], l[NT][2]; // of queries 2t, 2t+1: reference of the row sum, sum of the lane's own keys
  float top[NT][2];         // reference of the weights times their values' factors
  __device__ void clear() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = top[n][0] = top[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
    }
  }
  // Scores of keys g (s[..][0..1]) and g + 8 (s[..][2..3]) in log2 units, -infinity where there is no key, and the exponents
  // of their values -> the weights as the operand of O^T = V^T P^T.
  template <bool kBf16>
  __device__ __forceinline__ void weigh(const float (&s)[NT][4], float e0, float e1, uint32_t (&b)[NT][2]) {
    bool over = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        over = over || fmaxf(s[n][c], s[n][c + 2]) > m[n][c] + kFewSlack || fmaxf(s[n][c] + e0, s[n][c + 2] + e1) > top[n][c] + kFewSlack;
    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = fmaxf(s[n][c], s[n][c + 2]), y = fmaxf(s[n][c] + e0, s[n][c + 2] + e1);
#pragma unroll
          for (int d = 4; d < 32; d *= 2) {
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, d));
          }
          x = fmaxf(x, m[n][c]);
          y = fmaxf(y, top[n][c]);
          l[n][c] *= m[n][c] == -INFINITY ? 0.f : fast_exp2(m[n][c] - x);
          const float alpha = top[n][c] == -INFINITY ? 0.f : fast_exp2(top[n][c] - y);
          m[n][c] = x;
          top[n][c] = y;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            o[n][j][c] *= alpha;
            o[n][j][c + 2] *= alpha;
          }
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float w[4];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float ref = m[n][c] == -INFINITY ? 0.f : m[n][c], wref = (top[n][c] == -INFINITY ? 0.f : top[n][c]) - kFewBias;
        l[n][c] += fast_exp2(s[n][c] - ref) + fast_exp2(s[n][c + 2] - ref);
        w[c] = fast_exp2(s[n][c] + (e0 - wref));
        w[c + 2] = fast_exp2(s[n][c + 2] + (e1 - wref));
      }
      b[n][0] = transpose_8x8(kBf16 ? pack_bf16(w[0], w[1]) : pack_half(w[0], w[1]));
      b[n][1] = transpose_8x8(kBf16 ? pack_bf16(w[2], w[3]) : pack_half(w[2], w[3]));
    }
  }
};

// grid.x: (tile of 8 NT rows, split) with the split fastest, grid.y: head, grid.z: sample (one over a shared prefix).
template <int D, int NT>
__global__ void __launch_bounds__(FewShape<D, NT>::kThreads, 1) attn8_few_kernel(const FewArgs a) {
  using S = FewShape<D, NT>;
  constexpr int kFewWarps = S::kWarps, kFewThreads = S::kThreads;
  extern __shared__ __align__(16) uint8_t few_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % a.splits, row0 = blockIdx.x / a.splits * (8 * NT);
  const int h = blockIdx.y, bz = blockIdx.z;
  const long long list = static_cast<long long>(bz) * a.heads + h;
  const uint8_t* k_base = a.k + list * a.slot_tokens * D + t * 16;
  const uint8_t* v_base = a.v + list * a.slot_tokens * D + g * S::kVBytes;
  const uint8_t *ke = a.k_exp + list * a.slot_tokens, *ve = a.v_exp + list * a.slot_tokens;
  const uint32_t ring = smem_u32(few_smem) + warp * (S::kStages * S::kStageBytes);
  // row of the list -> sample and query
  auto sample_of = [&](int row) { return a.shared ? row / a.n_q : bz; };
  auto query_of = [&](int row) { return a.shared ? row % a.n_q : row; };

  // this CTA's steps: those of the cache first, then those of the chunks of the samples that the rows belong to
  const int row_end = min(row0 + 8 * NT, a.rows), first_sample = sample_of(row0);
  const int ctx_steps = (a.n_ctx + kFewStep - 1) / kFewStep, chunk_steps = (a.n_kc + kFewStep - 1) / kFewStep;
  const int steps = ctx_steps + (sample_of(row_end - 1) - first_sample + 1) * chunk_steps;
  const int each = steps / a.splits, rest = steps % a.splits;
  const int first = split * each + min(split, rest), last = first + each + (split < rest ? 1 : 0);
  const int ctx_last = min(last, ctx_steps);

  auto place = [&](int r) -> long long { return r < a.count0 ? a.start0 + r : a.start1 + (r - a.count0); };
  // keys behind the end: the last key's bytes, with a score of -infinity
  auto fetch = [&](int step, int stage) {
    if (step < ctx_last) {
      const int key0 = step * kFewStep;
      const uint32_t slot = ring + stage * S::kStageBytes + lane * 16;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* src = k_base + place(min(key0 + g + 8 * i, a.n_ctx - 1)) * D;
#pragma unroll
        for (int c = 0; c < S::kPieces; ++c) cp_async16(slot + (i * S::kPieces + c) * 512, src + c * 64);
      }
      const uint32_t v_slot = ring + stage * S::kStageBytes + 2 * S::kPieces * 512 + lane * S::kVBytes;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint8_t* src = v_base + place(min(key0 + 2 * t + (i & 1) + 8 * (i >> 1), a.n_ctx - 1)) * D;
        if constexpr (D == 128) cp_async16(v_slot + i * 512, src);
        else cp_async8(v_slot + i * 256, src);
      }
    }
    cp_async_commit();
  };
  uint32_t e_next[4];   // exponent bytes of keys g, g + 8: K, K, V, V
  auto fetch_exps = [&](int step) {
    if (step < ctx_last) {
      const long long r0 = place(min(step * kFewStep + g, a.n_ctx - 1)), r1 = place(min(step * kFewStep + g + 8, a.n_ctx - 1));
      e_next[0] = ke[r0]; e_next[1] = ke[r1]; e_next[2] = ve[r0]; e_next[3] = ve[r1];
    }
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) fetch(first + warp + i * kFewWarps, i);
  fetch_exps(first + warp);

  // Q in the order of the K pieces: elements 16 (t + 4 c) + 4 x + {0, 1} and {2, 3} of query 8 n + g
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
          const uint4 w = src[2 * (t + 4 * c) + x];
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

  int stage = 0;
  for (int step = first + warp; step < ctx_last; step += kFewWarps) {
    cp_async_wait<S::kStages - 2>();
    const uint4* slot = reinterpret_cast<const uint4*>(few_smem + warp * (S::kStages * S::kStageBytes) + stage * S::kStageBytes) + lane;
    const float ks0 = exp_byte_to_float(e_next[0]), ks1 = exp_byte_to_float(e_next[1]);
    const float vs0 = static_cast<float>(static_cast<int>(e_next[2]) - 127), vs1 = static_cast<float>(static_cast<int>(e_next[3]) - 127);
    fetch_exps(step + kFewWarps);
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
    for (int c = 0; c < S::kPieces; ++c) {
      const uint4 x = slot[c * 32], y = slot[(S::kPieces + c) * 32];
      const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a0 = e4m3_to_half2(xw[i]), a2 = e4m3_to_half2(xw[i] >> 16);
        const uint32_t a1 = e4m3_to_half2(yw[i]), a3 = e4m3_to_half2(yw[i] >> 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_16x8x16<false>(s[n], a0, a1, a2, a3, qf[n][c][i][0], qf[n][c][i][1]);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        s[n][c] *= ks0 * unit[n][c];
        s[n][c + 2] *= ks1 * unit[n][c];
      }
    const int left = a.n_ctx - step * kFewStep;   // keys from here to the end
    if (left < kFewStep) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (g + 8 * (e / 2) >= left) s[n][e] = -INFINITY;
    }
    uint32_t p[NT][2];
    st.template weigh<false>(s, vs0, vs1, p);
    // V: words of keys 2t, 2t+1, 2t+8, 2t+9
    uint32_t w[4][S::kVBytes / 4];
    const uint8_t* v_slot = few_smem + warp * (S::kStages * S::kStageBytes) + stage * S::kStageBytes + 2 * S::kPieces * 512 + lane * S::kVBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (D == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(v_slot + i * 512);
        w[i][0] = x.x; w[i][1] = x.y; w[i][2] = x.z; w[i][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(v_slot + i * 256);
        w[i][0] = x.x; w[i][1] = x.y;
      }
    }
#pragma unroll
    for (int i = 0; i < S::kVBytes / 4; ++i)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t sel = half ? 0x7362u : 0x5140u;   // codes of two elements, keys side by side
        const uint32_t x = __byte_perm(w[0][i], w[1][i], sel), y = __byte_perm(w[2][i], w[3][i], sel);
        const uint32_t a0 = e4m3_to_half2(x), a1 = e4m3_to_half2(x >> 16), a2 = e4m3_to_half2(y), a3 = e4m3_to_half2(y >> 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_16x8x16<false>(st.o[n][2 * i + half], a0, a1, a2, a3, p[n][0], p[n][1]);
      }
    int ahead = stage + S::kStages - 1;
    if (ahead >= S::kStages) ahead -= S::kStages;
    fetch(step + (S::kStages - 1) * kFewWarps, ahead);
    if (++stage == S::kStages) stage = 0;
  }

  // the chunks' own keys, bf16 [B, n_kc, H, D]; the warps take them in the order in which the cache's steps would have gone on
  int step = first + warp;
  if (step < ctx_steps) step += (ctx_steps - step + kFewWarps - 1) / kFewWarps * kFewWarps;
  if (step < last) load_q();
  for (; step < last; step += kFewWarps) {
    const int b = first_sample + (step - ctx_steps) / chunk_steps, key0 = (step - ctx_steps) % chunk_steps * kFewStep;
    auto row_of = [&](const __nv_bfloat16* base, int key) {
      return base + ((static_cast<long long>(b) * a.n_kc + min(key, a.n_kc - 1)) * a.heads + h) * D;
    };
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
    const uint4 *k0 = reinterpret_cast<const uint4*>(row_of(a.kc, key0 + g)), *k1 = reinterpret_cast<const uint4*>(row_of(a.kc, key0 + g + 8));
#pragma unroll
    for (int c = 0; c < S::kPieces; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 x = k0[2 * (t + 4 * c) + i], y = k1[2 * (t + 4 * c) + i];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_16x8x16<true>(s[n], x.x, y.x, x.y, y.y, qf[n][c][2 * i][0], qf[n][c][2 * i][1]);
          mma_16x8x16<true>(s[n], x.z, y.z, x.w, y.w, qf[n][c][2 * i + 1][0], qf[n][c][2 * i + 1][1]);
        }
      }
    const int left = a.n_kc - key0;
    // a sample's keys are seen by its own queries
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[n][e] = g + 8 * (e / 2) < left && sample_of(row0 + 8 * n + 2 * t + e % 2) == b ? s[n][e] * a.scale_log2 : -INFINITY;
    // no weight for those who do not see the key, whatever its value holds: 0 * NaN would reach them
    uint32_t p[NT][2];
    st.template weigh<true>(s, 0.f, 0.f, p);
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
                            __byte_perm(w[2][j], w[3][j], 0x5410), __byte_perm(w[2][j], w[3][j], 0x7632), p[n][0], p[n][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (sample_of(row0 + 8 * n + 2 * t + e % 2) == b) st.o[n][4 * i + j][e] += add[e];
        }
    }
  }

  // ---- the warps' outputs joined: [warp][query][D], then [warp][query] of references and sums
  cp_async_wait<0>();
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
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) top = fmaxf(top, stats[w * 8 * NT + i].x);
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float4 f = stats[w * 8 * NT + i];
      const float2 v = *reinterpret_cast<const float2*>(out + (w * 8 * NT + i) * D + d);
      const float weight = fast_exp2(f.z - kFewBias - ref);   // 0 for a warp without keys, here and next
      l = fmaf(fast_exp2(f.x - ref), f.y, l);
      o0 = fmaf(weight, v.x, o0);
      o1 = fmaf(weight, v.y, o1);
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
  dependents_may_start();
}
template <int D, int NT> constexpr int few_smem_bytes() {
  const int joined = FewShape<D, NT>::kWarps * 8 * NT * (D + 4) * 4;
  return FewShape<D, NT>::kRing > joined ? FewShape<D, NT>::kRing : joined;
}

}  // namespace astro
