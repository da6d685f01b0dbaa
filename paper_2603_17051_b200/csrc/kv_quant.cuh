// The rolling cache in 8 bits.  A row x (the D elements of one head and token) is held as one exponent e and D codes:
//   e = the smallest whole number with max |x_d| <= 448 * 2^e over the row's finite elements, at least -124;
//   code_d = e4m3(x_d * 2^-e), rounded to nearest even; an infinity or NaN becomes e4m3's NaN and touches no other element.
//   (Of rows beyond 1.75 * 2^127 e is 120, and elements that would round to 256 * 2^120, beyond every finite float, are held as 240.)
// The factor is a power of two, so that what a code stands for, code * 2^e, has 4 significant bits and a step of 2^-133 or
// more: it is a bf16 number exactly, and attention over it needs no rounding beyond the one that the write made (half a step
// of e4m3, 2^-4 of the element, or 2^(e-10) where that is larger).
// Storage: codes [B_c, H, slot * T + t, D], then, from the next multiple of 16 bytes on, e + 127 as a byte for every row.
// Everything here is bandwidth work: a thread owns 8 neighbouring elements (16 bytes of bf16, 8 of codes) of one head and walks
// kQuantTokens tokens, all of them in flight, so that a warp reads 512 contiguous bytes of the caller's tensor and writes whole rows.
// 3 frames of 1560 tokens, 12 heads of 128, 4 samples, bf16: written in 35 us (174 MB, 4.9 TB/s: 2.9 instructions a clock, the row's
// maximum and the conversions; 119 us when each element was tested for being finite on its own), read back in 27 (174 MB, 6.5 TB/s).
// 18 frames of one sample read back in 41.5 us: 260 MB at 6.25 TB/s, 95 % of a plain copy.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace astro {

constexpr int kQuantTokens = 8;
constexpr int kQuantThreads = 256;
constexpr int kQuantLowestExp = -124;

// Where the frames of a call sit: frame j of the call is the cache's logical frame first + j; the sink's frames sit in their
// own slots, the window's in the ring behind them.
struct FrameSlots {
  int first, sink_frames, sink_held, win_head, win_slots;
  __host__ __device__ int slot(int j) const {
    const int f = first + j;
    if (f < sink_held) return f;
    const unsigned at = static_cast<unsigned>(win_head) + static_cast<unsigned>(f - sink_held);   // less than two rounds
    return sink_frames + static_cast<int>(at < static_cast<unsigned>(win_slots) ? at : at - win_slots);
  }
};

struct QuantTensors {
  void *k, *v;                       // the caller's
  uint8_t *k_store, *v_store;        // codes
  uint8_t *k_exp, *v_exp;
  long long in_b, in_t, in_h;        // strides of the caller's tensors in elements
  long long slot_tokens;             // tokens of the storage per (sample, head)
  int heads, tokens_per_frame, n_tokens;
};

// 8 neighbouring elements as they come, and in fp32.
template <typename T> struct Raw8 {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* p) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    if constexpr (sizeof(T) == 4) {
      const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
      w[4] = u.x; w[5] = u.y; w[6] = u.z; w[7] = u.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 2 * static_cast<int>(sizeof(T)); ++i) w[i] = 0;
  }
  __device__ __forceinline__ float2 pair(int i) const {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else if constexpr (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    else return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  // The largest magnitude's bits as those of a float, infinities and NaN left out.
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
    if constexpr (sizeof(T) == 2) {
      constexpr bool kHalf = std::is_same<T, __half>::value;
      constexpr uint32_t kInf = kHalf ? 0x7c00u : 0x7f80u;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);   // magnitudes are ordered like their bits
      m = max(m >> 16, m & 0xffffu);
      if (m >= kInf) {                                  // rare
        m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t x = (w[i / 2] >> (16 * (i & 1))) & 0x7fffu;
          m = max(m, x < kInf ? x : 0u);
        }
      }
      if constexpr (kHalf) return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(m))));
      else return m << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t x = w[i] & 0x7fffffffu;
        m = max(m, x < 0x7f800000u ? x : 0u);
      }
      return m;
    }
  }
};
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Two floats of at most 448 in magnitude (or NaN) -> two e4m3 codes, `lo` in the low byte.
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two codes in the low 16 bits -> two fp16, which hold every e4m3 number (and its NaN).
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(codes)));
  return r;
}
__device__ __forceinline__ float2 e4m3_to_floats(uint32_t codes) {
  const uint32_t h = e4m3_to_half2(codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// 2^e of a stored exponent byte (3..247): its own exponent field.
__device__ __forceinline__ float exp_byte_to_float(uint32_t byte) { return __uint_as_float(byte << 23); }

// The lanes of a row each hold a value for every token; afterwards lane x holds the maximum over them for token x % kQuantTokens:
// they halve the tokens among themselves step by step instead of every lane learning every token's.
template <int kLanes>
__device__ __forceinline__ uint32_t max_per_token(uint32_t (&v)[kQuantTokens], int lane) {
  static_assert(kQuantTokens == 8 && (kLanes == 8 || kLanes == 16), "three halvings, and one more step over 16 lanes");
#pragma unroll
  for (int half = 4; half > 0; half /= 2) {
    const bool upper = lane & half;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const uint32_t give = upper ? v[i] : v[i + half], keep = upper ? v[i + half] : v[i];
      v[i] = max(keep, __shfl_xor_sync(0xffffffffu, give, half));
    }
  }
  if constexpr (kLanes == 16) v[0] = max(v[0], __shfl_xor_sync(0xffffffffu, v[0], 8));
  return v[0];
}

// grid.x: token chunks, grid.y: head * D/8 positions, grid.z = 2 * b + (0: K, 1: V).  Lanes without a position stay for the
// shuffles.
template <typename T, int D>
__global__ void __launch_bounds__(kQuantThreads) cache8_append_kernel(const QuantTensors x, const FrameSlots slots) {
  constexpr int kLanes = D / 8;                         // lanes of a row
  const int hv = blockIdx.y * blockDim.x + threadIdx.x, lane = threadIdx.x & 31;
  const bool there = hv < x.heads * kLanes;
  const int h = there ? hv / kLanes : 0, part = hv % kLanes;
  const int b = blockIdx.z >> 1;
  const bool is_v = blockIdx.z & 1;
  const int t0 = blockIdx.x * kQuantTokens;
  const int n = there ? min(kQuantTokens, x.n_tokens - t0) : 0;
  const T* src = static_cast<const T*>(is_v ? x.v : x.k) + b * x.in_b + t0 * x.in_t + h * x.in_h + part * 8;
  Raw8<T> f[kQuantTokens];
#pragma unroll
  for (int i = 0; i < kQuantTokens; ++i) {
    if (i < n) f[i].load(src + i * x.in_t);
    else f[i].clear();
  }
  const long long row_base = (static_cast<long long>(b) * x.heads + h) * x.slot_tokens;
  uint8_t* codes = is_v ? x.v_store : x.k_store;
  uint8_t* exps = is_v ? x.v_exp : x.k_exp;
  int frame = t0 / x.tokens_per_frame;
  const int in_frame = t0 - frame * x.tokens_per_frame;
  // where token i of these goes; most often all of them are in one frame
  const long long row0 = row_base + static_cast<long long>(slots.slot(frame)) * x.tokens_per_frame + in_frame;
  const bool one_frame = in_frame + kQuantTokens <= x.tokens_per_frame;
  auto row_of = [&](int i) -> long long {
    if (one_frame) return row0 + i;
    const int fr = (t0 + i) / x.tokens_per_frame;
    return row_base + static_cast<long long>(slots.slot(fr)) * x.tokens_per_frame + (t0 + i - fr * x.tokens_per_frame);
  };
  uint32_t tops[kQuantTokens];
#pragma unroll
  for (int i = 0; i < kQuantTokens; ++i) tops[i] = f[i].top();
  const uint32_t top = max_per_token<kLanes>(tops, lane);
  // top = 1.f * 2^k <= 1.75 * 2^(e + 8)
  const int k = static_cast<int>(top >> 23) - 127;
  const int my_e = max(kQuantLowestExp, k - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0));
  if (part < kQuantTokens && part < n) exps[row_of(part)] = static_cast<uint8_t>(my_e + 127);
#pragma unroll
  for (int i = 0; i < kQuantTokens; ++i) {
    const int e = __shfl_sync(0xffffffffu, my_e, (lane & ~(kLanes - 1)) + i);
    const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);   // 2^-e: -e is 124 at most, -120 at least
    const float most = e == 120 ? 240.f : 448.f;
    uint32_t w[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      float y[4];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float2 v = f[i].pair(2 * p + c);
        // an infinity becomes NaN (0 * infinity), a finite number is left as it is
        y[2 * c] = fminf(fmaxf(v.x * inv, -most), most) + 0.f * v.x;
        y[2 * c + 1] = fminf(fmaxf(v.y * inv, -most), most) + 0.f * v.y;
      }
      w[p] = e4m3_pair(y[0], y[1]) | e4m3_pair(y[2], y[3]) << 16;
    }
    if (i < n) *reinterpret_cast<uint2*>(codes + row_of(i) * D + part * 8) = make_uint2(w[0], w[1]);
  }
}

// The reverse, into contiguous rows at strides of the caller's (in_b, in_t, in_h).  The same grid.
template <typename T, int D>
__global__ void __launch_bounds__(kQuantThreads) cache8_read_kernel(const QuantTensors x, const FrameSlots slots) {
  constexpr int kLanes = D / 8;
  const int hv = blockIdx.y * blockDim.x + threadIdx.x;
  if (hv >= x.heads * kLanes) return;
  const int h = hv / kLanes, part = hv % kLanes;
  const int b = blockIdx.z >> 1;
  const bool is_v = blockIdx.z & 1;
  const int t0 = blockIdx.x * kQuantTokens;
  const int n = min(kQuantTokens, x.n_tokens - t0);
  const long long row_base = (static_cast<long long>(b) * x.heads + h) * x.slot_tokens;
  const uint8_t* codes = is_v ? x.v_store : x.k_store;
  const uint8_t* exps = is_v ? x.v_exp : x.k_exp;
  int frame = t0 / x.tokens_per_frame, in_frame = t0 - frame * x.tokens_per_frame;
  long long slot_row = row_base + static_cast<long long>(slots.slot(frame)) * x.tokens_per_frame;
  uint2 w[kQuantTokens];
  uint32_t e[kQuantTokens];
#pragma unroll
  for (int i = 0; i < kQuantTokens; ++i) {
    if (i >= n) continue;
    const long long row = slot_row + in_frame;
    w[i] = *reinterpret_cast<const uint2*>(codes + row * D + part * 8);
    e[i] = exps[row];
    if (++in_frame == x.tokens_per_frame) {
      in_frame = 0;
      if (i + 1 < n) slot_row = row_base + static_cast<long long>(slots.slot(++frame)) * x.tokens_per_frame;
    }
  }
  T* dst = static_cast<T*>(is_v ? x.v : x.k) + b * x.in_b + t0 * x.in_t + h * x.in_h + part * 8;
#pragma unroll
  for (int i = 0; i < kQuantTokens; ++i) {
    if (i >= n) continue;
    const float s = exp_byte_to_float(e[i]);
    const float2 p[4] = {e4m3_to_floats(w[i].x), e4m3_to_floats(w[i].x >> 16), e4m3_to_floats(w[i].y), e4m3_to_floats(w[i].y >> 16)};
    float f[8];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      f[2 * c] = p[c].x * s;
      f[2 * c + 1] = p[c].y * s;
    }
    store8(dst + i * x.in_t, f);
  }
}

// Exponent bytes of frames copied into another cache (fork; the codes go the way of every cache's bytes): frame first_to + j of
// sample b takes slot from.slot[j] of sample parents[b].  A parent outside the source leaves zeros, whose rows stand for zeros.
// grid.x = ((frame, head) * 2 + (0: K, 1: V)) * batch + b
struct ForkSlots {
  int from[32];
  int first_to;
};
__global__ void __launch_bounds__(128)
cache8_fork_exps_kernel(const uint8_t* __restrict__ k_src, const uint8_t* __restrict__ v_src, uint8_t* __restrict__ k_dst,
                        uint8_t* __restrict__ v_dst, const int* __restrict__ parents, const ForkSlots slots, const int source_batch,
                        const int batch, const int heads, const int tokens_per_frame, const int src_slots, const int dst_slots) {
  unsigned i = blockIdx.x;
  const int b = i % batch;
  i /= batch;
  const bool is_v = i & 1;
  i >>= 1;
  const int h = i % heads, j = i / heads;
  const int parent = parents ? parents[b] : (source_batch == 1 ? 0 : b);
  const bool there = parent >= 0 && parent < source_batch;
  const uint8_t* src = (is_v ? v_src : k_src) +
                       ((static_cast<long long>(there ? parent : 0) * heads + h) * src_slots + slots.from[j]) * tokens_per_frame;
  uint8_t* dst = (is_v ? v_dst : k_dst) + ((static_cast<long long>(b) * heads + h) * dst_slots + slots.first_to + j) * tokens_per_frame;
  for (int t = threadIdx.x; t < tokens_per_frame; t += 128) dst[t] = there ? src[t] : 0;
}

}  // namespace astro
