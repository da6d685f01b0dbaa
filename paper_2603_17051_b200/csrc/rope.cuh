// Rotary positions of queries and keys, forward and transposed (the backward pass).
//   pair p of token t turns by the angle  x = coordinate[t, axis(p)] * f_p:
//   (a, b) -> size * (a cos x - b sin x, a sin x + b cos x);  transposed: sin x -> -sin x.
// Pairs are neighbours (2p, 2p + 1) or halves (p, p + rot/2); elements from rot_dim on are copied.
//
// Angles: coordinate * (f_p / 2 pi) is formed in fp64 and reduced to a fraction of a turn there, so that far
// positions lose nothing (an fp32 product is 0.06 rad off at position 10^6); sine and cosine of the fraction are
// fp32 (2e-7 rad), the rotation is fp32 and each result is rounded once to the tensor's type.
//
// The work is bandwidth: q and k read once, written once.  A thread owns one 16-byte piece of a token's rows (two where
// pairs are halves), works out the cosines and sines of its 2 to 8 pairs itself and walks over the rows (the heads of q, then
// those of k), kRopeRows loads in flight: no shared memory, no barrier, and the angles cost a fifth of the instructions when a thread
// has all 24 rows of a 12-head token.  With fewer tokens the rows are dealt to several threads.
// Halves whose half is no multiple of 16 bytes take one pair of single elements per thread and row, nothing asked for ahead: 27 us for the
// same tensors with 124 of 128 elements turning.
// Sharing the angles of a few tokens through shared memory instead made every block load, wait, turn and store in step: 18.4 us
// against 12.1 us for the 4680 tokens of a chunk (57.6 MB).  fp32, 8 samples (920 MB): 140 us = 6.6 TB/s, the copy rate.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace astro {

constexpr int kRopeMaxPairs = 128;
constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 6;        // rows whose loads a thread has in flight

struct RopeTable {
  double turns[kRopeMaxPairs];      // f_p / 2 pi
  uint8_t axis[kRopeMaxPairs];
  float size;
  int pairs, axes;
};

struct RopeTensors {
  const void *q, *k;   // k null: q alone
  void *q_out, *k_out;
  long long in_b, in_t, in_h, out_b, out_t, out_h;   // strides in elements
  int heads_q, heads_k;
};

template <typename T> struct RopeVec;
template <> struct RopeVec<__nv_bfloat16> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = __bfloat1622float2(p[i]); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint4 v;
    __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    return v;
  }
  static __device__ __forceinline__ float load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, float f) { *p = __float2bfloat16_rn(f); }
};
template <> struct RopeVec<__half> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const __half2* p = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(p[i]); f[2 * i] = x.x; f[2 * i + 1] = x.y; }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint4 v;
    __half2* p = reinterpret_cast<__half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    return v;
  }
  static __device__ __forceinline__ float load(const __half* p) { return __half2float(*p); }
  static __device__ __forceinline__ void store(__half* p, float f) { *p = __float2half_rn(f); }
};
template <> struct RopeVec<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float f) { *p = f; }
};

// How a thread's work on a row is cut: 0 neighbouring pairs, 16 bytes per item; 1 halves whose two 16-byte pieces
// both start on 16 bytes (half the rotated part is a multiple of 16 bytes); 2 halves otherwise, one pair of single
// elements per item.
enum { kRopeInterleaved = 0, kRopeHalves = 1, kRopeHalvesScalar = 2 };

__host__ __device__ inline int rope_items_per_row(int mode, int head_dim, int rot_dim, int elems) {
  if (mode == kRopeInterleaved) return head_dim / elems;
  if (mode == kRopeHalves) return rot_dim / 2 / elems + (head_dim - rot_dim) / elems;
  return rot_dim / 2 + (head_dim - rot_dim);
}

// Thread = (token, row phase, item): the rows phase, phase + phases, ... of the token.  Tokens are numbered sample-major,
// batch * n_tokens in all.
template <typename T, int MODE>
__global__ void __launch_bounds__(kRopeThreads)
rope_kernel(const __grid_constant__ RopeTable table, const __grid_constant__ RopeTensors x,
            const int* __restrict__ positions, const int positions_per_sample, const int n_tokens, const int total_tokens,
            const int head_dim, const int rot_dim, const int phases, const float sign) {
  constexpr int E = RopeVec<T>::kElems;
  constexpr int kPairs = MODE == kRopeInterleaved ? E / 2 : MODE == kRopeHalves ? E : 1;   // pairs of an item
  const int per_row = rope_items_per_row(MODE, head_dim, rot_dim, E);
  const long long id = static_cast<long long>(blockIdx.x) * kRopeThreads + threadIdx.x;
  const int token = static_cast<int>(id / (per_row * phases));
  if (token >= total_tokens) return;
  const int rest = static_cast<int>(id - static_cast<long long>(token) * (per_row * phases));
  const int phase = rest / per_row, c = rest - phase * per_row;
  const int b = token / n_tokens, t = token - b * n_tokens;
  const int half = rot_dim / 2;
  // first pair of the item, how many of its pairs turn, its first element
  const int p0 = c * kPairs;
  const int turning = min(kPairs, max(0, half - p0));
  const int e0 = MODE == kRopeInterleaved ? c * E : turning > 0 ? p0 : p0 + half;   // copied pieces of halves start at rot_dim

  const int rows = x.heads_q + x.heads_k;
  const long long in0 = b * x.in_b + t * x.in_t + e0, out0 = b * x.out_b + t * x.out_t + e0;
  auto source = [&](int r) {
    return r < x.heads_q ? static_cast<const T*>(x.q) + in0 + r * x.in_h
                         : static_cast<const T*>(x.k) + in0 + (r - x.heads_q) * x.in_h;
  };
  auto target = [&](int r) {
    return r < x.heads_q ? static_cast<T*>(x.q_out) + out0 + r * x.out_h
                         : static_cast<T*>(x.k_out) + out0 + (r - x.heads_q) * x.out_h;
  };
  // the piece, and its partner half a rotated part further on
  uint4 v[kRopeRows], w[MODE == kRopeHalves ? kRopeRows : 1];
  auto fetch = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kRopeRows; ++u) {
      const int r = r0 + u * phases;
      if (r >= rows) continue;
      const T* src = source(r);
      v[u] = __ldcs(reinterpret_cast<const uint4*>(src));
      if (MODE == kRopeHalves && turning > 0) w[u] = __ldcs(reinterpret_cast<const uint4*>(src + half));
    }
  };
  if (MODE != kRopeHalvesScalar) fetch(phase);   // on their way while the angles are worked out

  float cs[kPairs], sn[kPairs];
  const int* coordinate = positions + static_cast<long long>(positions_per_sample ? token : t) * table.axes;
#pragma unroll
  for (int j = 0; j < kPairs; ++j)
    if (j < turning) {
      double turns = static_cast<double>(coordinate[table.axis[p0 + j]]) * table.turns[p0 + j];
      turns -= rint(turns);
      sincospif(2.f * static_cast<float>(turns), &sn[j], &cs[j]);
      cs[j] *= table.size;
      sn[j] *= table.size * sign;
    }

  if constexpr (MODE == kRopeHalvesScalar) {
    for (int r = phase; r < rows; r += phases) {
      const T* src = source(r);
      T* dst = target(r);
      if (turning == 0) {
        *dst = *src;
        continue;
      }
      const float lo = RopeVec<T>::load(src), hi = RopeVec<T>::load(src + half);
      RopeVec<T>::store(dst, lo * cs[0] - hi * sn[0]);
      RopeVec<T>::store(dst + half, lo * sn[0] + hi * cs[0]);
    }
  } else {
    for (int r0 = phase; r0 < rows;) {
#pragma unroll
      for (int u = 0; u < kRopeRows; ++u) {
        const int r = r0 + u * phases;
        if (r >= rows) continue;
        T* dst = target(r);
        if (turning == 0) {   // stored bit for bit as it came
          __stcs(reinterpret_cast<uint4*>(dst), v[u]);
        } else if (MODE == kRopeInterleaved) {
          float f[E];
          RopeVec<T>::unpack(v[u], f);
#pragma unroll
          for (int j = 0; j < kPairs; ++j)
            if (j < turning) {
              const float lo = f[2 * j], hi = f[2 * j + 1];
              f[2 * j] = lo * cs[j] - hi * sn[j];
              f[2 * j + 1] = lo * sn[j] + hi * cs[j];
            }
          __stcs(reinterpret_cast<uint4*>(dst), RopeVec<T>::pack(f));
        } else {
          float lo[E], hi[E];
          RopeVec<T>::unpack(v[u], lo);
          RopeVec<T>::unpack(w[u], hi);
#pragma unroll
          for (int j = 0; j < E; ++j) {   // half is a multiple of E: the whole piece turns
            const float a = lo[j] * cs[j % kPairs] - hi[j] * sn[j % kPairs];
            hi[j] = lo[j] * sn[j % kPairs] + hi[j] * cs[j % kPairs];
            lo[j] = a;
          }
          __stcs(reinterpret_cast<uint4*>(dst), RopeVec<T>::pack(lo));
          __stcs(reinterpret_cast<uint4*>(dst + half), RopeVec<T>::pack(hi));
        }
      }
      r0 += kRopeRows * phases;
      if (r0 < rows) fetch(r0);
    }
  }
}

}  // namespace astro
