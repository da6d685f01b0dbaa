// Rotary positions of queries and keys, forward and transposed (the backward pass).
//   pair p of token t turns by the angle  x = coordinate[t, axis(p)] * f_p:
//   (a, b) -> size * (a cos x - b sin x, a sin x + b cos x);  transposed: sin x -> -sin x.
// Pairs are neighbours (2p, 2p + 1) or halves (p, p + rot/2); elements from rot_dim on are copied.
//
// Angles: coordinate * (f_p / 2 pi) is formed in fp64 and reduced to a fraction of a turn there, so that far
// positions lose nothing (an fp32 product is 0.06 rad off at position 10^6); sine and cosine of the fraction are
// fp32 (2e-7 rad), the rotation is fp32 and each result is rounded once to the tensor's type.
//
// The work is bandwidth: q and k read once, written once.  A block owns a few tokens: its threads first compute the
// tokens' cosines and sines into shared memory (once for all heads of q and k), then every thread keeps one 16-byte
// position of a token's rows and walks over the tokens, so that up to four loads per thread are in flight and no
// index is divided inside the loop.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace astro {

constexpr int kRopeMaxPairs = 128;
constexpr int kRopeMaxThreads = 512;
constexpr int kRopeUnroll = 4;      // tokens whose loads a thread has in flight
constexpr int kRopeMaxTokens = 32;  // tokens of a block

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

// blockDim.x threads share a token's (row, item) positions, blockDim.y token lanes; a block owns
// `block_tokens` consecutive tokens of the batch * n_tokens (sample-major).  Shared memory: float2 [tokens][pairs].
template <typename T, int MODE>
__global__ void __launch_bounds__(kRopeMaxThreads)
rope_kernel(const __grid_constant__ RopeTable table, const __grid_constant__ RopeTensors x,
            const int* __restrict__ positions, const int positions_per_sample, const int n_tokens, const int total_tokens,
            const int head_dim, const int rot_dim, const int block_tokens, const float sign) {
  constexpr int E = RopeVec<T>::kElems;
  extern __shared__ float2 s_turn[];
  __shared__ long long s_in[kRopeMaxTokens], s_out[kRopeMaxTokens];
  const int first = blockIdx.x * block_tokens;
  const int count = min(block_tokens, total_tokens - first);
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
  for (int i = tid; i < count * table.pairs; i += threads) {
    const int t = i / table.pairs, p = i - t * table.pairs;
    const long long row = positions_per_sample ? first + t : (first + t) % n_tokens;
    double turn = static_cast<double>(positions[row * table.axes + table.axis[p]]) * table.turns[p];
    turn -= rint(turn);
    float sn, cs;
    sincospif(2.f * static_cast<float>(turn), &sn, &cs);
    s_turn[i] = make_float2(cs * table.size, sn * table.size * sign);
  }
  if (tid < count) {
    const int b = (first + tid) / n_tokens, t = (first + tid) - b * n_tokens;
    s_in[tid] = b * x.in_b + t * x.in_t;
    s_out[tid] = b * x.out_b + t * x.out_t;
  }
  __syncthreads();

  const int per_row = rope_items_per_row(MODE, head_dim, rot_dim, E);
  const int items = (x.heads_q + x.heads_k) * per_row;
  const int half = rot_dim / 2;
  for (int i = threadIdx.x; i < items; i += blockDim.x) {
    const int r = i / per_row, c = i - r * per_row;
    const bool is_k = r >= x.heads_q;
    const int h = is_k ? r - x.heads_q : r;
    const T* in = static_cast<const T*>(is_k ? x.k : x.q) + h * x.in_h;
    T* out = static_cast<T*>(is_k ? x.k_out : x.q_out) + h * x.out_h;
    if (MODE == kRopeInterleaved) {
      const int e0 = c * E, p0 = e0 / 2, rotated = min(E / 2, max(0, half - p0));
      for (int t0 = threadIdx.y; t0 < count; t0 += kRopeUnroll * blockDim.y) {
        uint4 v[kRopeUnroll];
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
          const int t = t0 + u * blockDim.y;
          if (t < count) v[u] = *reinterpret_cast<const uint4*>(in + s_in[t] + e0);
        }
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
          const int t = t0 + u * blockDim.y;
          if (t >= count) break;
          float f[E];
          RopeVec<T>::unpack(v[u], f);
          const float2* cs = s_turn + t * table.pairs + p0;
#pragma unroll
          for (int j = 0; j < E / 2; ++j)
            if (j < rotated) {
              const float2 w = cs[j];
              const float a = f[2 * j], b = f[2 * j + 1];
              f[2 * j] = a * w.x - b * w.y;
              f[2 * j + 1] = a * w.y + b * w.x;
            }
          // a piece without rotated elements is stored bit for bit as it came
          *reinterpret_cast<uint4*>(out + s_out[t] + e0) = rotated == 0 ? v[u] : RopeVec<T>::pack(f);
        }
      }
    } else if (MODE == kRopeHalves) {
      const bool copy = c >= half / E;
      const int e0 = copy ? c * E + half : c * E;   // copied pieces start at rot_dim
      for (int t0 = threadIdx.y; t0 < count; t0 += kRopeUnroll * blockDim.y) {
        uint4 v[kRopeUnroll], w[kRopeUnroll];
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
          const int t = t0 + u * blockDim.y;
          if (t >= count) continue;
          v[u] = *reinterpret_cast<const uint4*>(in + s_in[t] + e0);
          if (!copy) w[u] = *reinterpret_cast<const uint4*>(in + s_in[t] + e0 + half);
        }
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) {
          const int t = t0 + u * blockDim.y;
          if (t >= count) continue;
          if (copy) {
            *reinterpret_cast<uint4*>(out + s_out[t] + e0) = v[u];
            continue;
          }
          float a[E], b[E];
          RopeVec<T>::unpack(v[u], a);
          RopeVec<T>::unpack(w[u], b);
          const float2* cs = s_turn + t * table.pairs + e0;
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float2 y = cs[j];
            const float lo = a[j] * y.x - b[j] * y.y;
            b[j] = a[j] * y.y + b[j] * y.x;
            a[j] = lo;
          }
          *reinterpret_cast<uint4*>(out + s_out[t] + e0) = RopeVec<T>::pack(a);
          *reinterpret_cast<uint4*>(out + s_out[t] + e0 + half) = RopeVec<T>::pack(b);
        }
      }
    } else {
      const bool copy = c >= half;
      const int e0 = copy ? c + half : c;
      for (int t = threadIdx.y; t < count; t += blockDim.y) {
        const T* src = in + s_in[t] + e0;
        T* dst = out + s_out[t] + e0;
        if (copy) {
          *dst = *src;
          continue;
        }
        const float a = RopeVec<T>::load(src), b = RopeVec<T>::load(src + half);
        const float2 y = s_turn[t * table.pairs + c];
        RopeVec<T>::store(dst, a * y.x - b * y.y);
        RopeVec<T>::store(dst + half, a * y.y + b * y.x);
      }
    }
  }
}

}  // namespace astro
