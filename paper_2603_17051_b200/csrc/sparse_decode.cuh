// Forward of attention over lists of key blocks for one or two queries per sample: the form of single-token decoding.
//
// A list is read once and every key meets one or two queries: bandwidth, 2 * keys * D * 2 bytes per query list.  An MMA tile
// would be 1/128 full and its softmax, bound to the quarter of tensor memory that holds the query's row, would run on one
// of the SM's four schedulers (32 us for 4 x 12 lists of 3840 keys, of which the bytes are 14.4).  So the arithmetic is
// done by the ordinary cores, in fp32 from the bf16 values, P included: 20.5 us, 94 MB from DRAM; longer lists add
// their bytes at 5.9 to 6.2 TB/s.  Two queries of head_dim 128 keep 31 words per thread in local memory (168
// registers are the most that 320 threads get): about 30 reloads per warp and tile, 4 % of the instructions.
//
// A cluster of up to 8 CTAs shares a list, each CTA walks over its range of it: two warps follow the list and load the key
// tiles (the same boxes as the MMA kernel's), one K, one V, into rings of three; the other warps compute.  A warp owns 8 or
// 16 keys of every tile and its own running maximum, sum and output: four or two lanes per key for the scores, then eight
// columns per lane for the output, the weights coming by shuffles; so warps never wait for each other inside the loop.  At
// the end the warps' outputs are joined in shared memory, the CTAs' through distributed shared memory: no second launch, no
// scratch.  The order in which lanes read follows the tiles' swizzle so that no two lanes of a quarter warp meet in a bank.
#pragma once
#include "sparse_common.cuh"

namespace astro {

constexpr int kDecodeStages = 3;
constexpr int kDecodeMaxQueries = 2, kDecodeMaxCluster = 8;
// Computing warps: 16 for one query; two queries need twice the registers per thread.
template <int R> struct DecodeShape {
  static constexpr int kWarps = R == 1 ? 16 : 8;
  static constexpr int kThreads = 32 * kWarps + 64;
  static constexpr int kKeys = kTile / kWarps;      // keys of a warp per tile
};

template <int D, int R> struct DecodeSmem {
  static constexpr int kK = 0;
  static constexpr int kV = kDecodeStages * TileGeom<D>::kBytes;
  static constexpr int kOut = 2 * kDecodeStages * TileGeom<D>::kBytes;                       // float [warps][queries][D]
  static constexpr int kStats = kOut + DecodeShape<R>::kWarps * R * D * 4;                   // float [warps][queries][2]
  static constexpr int kJoined = kStats + DecodeShape<R>::kWarps * R * 8;                    // float [queries][2]: the CTA's
  static constexpr int kBars = kJoined + R * 8;
  static constexpr int kSource = kBars + 4 * kDecodeStages * 8 + 16;                         // of the K and of the V warp
  static constexpr int kDesc = kSource + 2 * static_cast<int>(sizeof(TileSource));           // per stage
  static constexpr int kTotal = kDesc + kDecodeStages * static_cast<int>(sizeof(TileDesc)) + 1024;
};

struct DecodeArgs {
  const __nv_bfloat16* q;
  const int* blocks;
  __nv_bfloat16* o;
  float* lse;
  int heads, n_select, entries, cache_shared;   // entries: list entries per CTA of the cluster
  float scale_log2;
};

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
// 16-byte piece `piece` (0 .. D/8 - 1) of row `row` of a tile
__device__ __forceinline__ uint4 tile_piece(const uint8_t* tile, int row, int piece) {
  return *reinterpret_cast<const uint4*>(tile + (piece >> 3) * (kTile * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

// The c-th 16-byte piece of a row that lane part `sub` of `lanes` reads for the scores.  In one step the eight lanes of a
// quarter warp read 8 / lanes neighbouring rows; their pieces fall into eight different places of the 128-byte swizzle.
template <int D> __device__ __forceinline__ int score_piece(int lanes, int sub, int c) {
  const int n = D / 8 / lanes;
  if (D == 64) return sub * n + c;
  return lanes == 2 ? sub * 8 + ((c + sub * 4) & 7) : sub * 4 + ((c + (sub >> 1) * 2) & 3);
}

// grid = (cluster size, heads, batch); R = queries per sample.
template <int D, int R>
__global__ void __launch_bounds__(DecodeShape<R>::kThreads, 1)
sparse_decode_kernel(const __grid_constant__ SparseMaps maps, const __grid_constant__ DecodeArgs a,
                     const __grid_constant__ SparseGeom g) {
  constexpr int kWarps = DecodeShape<R>::kWarps, kThreads = DecodeShape<R>::kThreads, kKeys = DecodeShape<R>::kKeys;
  using Smem = DecodeSmem<D, R>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align_1024(smem_raw);
  uint8_t *sK = smem + Smem::kK, *sV = smem + Smem::kV;
  float* s_out = reinterpret_cast<float*>(smem + Smem::kOut);
  float* s_stat = reinterpret_cast<float*>(smem + Smem::kStats);
  uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + Smem::kBars);
  uint64_t *k_empty = k_full + kDecodeStages, *v_full = k_empty + kDecodeStages, *v_empty = v_full + kDecodeStages;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(v_empty + kDecodeStages);
  TileDesc* desc = reinterpret_cast<TileDesc*>(smem + Smem::kDesc);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int parts = gridDim.x, part = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int from = part * a.entries, count = max(0, min(a.entries, a.n_select - from));
  const int* list = a.blocks + (static_cast<long long>(b) * a.heads + h) * a.n_select + from;

  int first = -1;
  if (warp >= kWarps) {
    first = ListWalker::first_entries(list, count, lane);
    if (lane == 0) {
      tma_prefetch_desc(warp == kWarps ? &maps.kx : &maps.vx);
      tma_prefetch_desc(warp == kWarps ? &maps.kc : &maps.vc);
    }
  }
  if (tid == 0) {
    for (int i = 0; i < kDecodeStages; ++i) {
      mbar_init(k_full + i, 1);
      mbar_init(v_full + i, 1);
      mbar_init(k_empty + i, kWarps);
      mbar_init(v_empty + i, kWarps);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  zero_uncovered_rows<D>(sK, 2 * kDecodeStages, g, tid, kThreads);   // K and V stages follow each other
  fence_proxy_async_smem();
  __syncthreads();

  if (warp >= kWarps) {
    const bool is_k = warp == kWarps;
    uint8_t* ring = is_k ? sK : sV;
    uint64_t *full = is_k ? k_full : v_full, *empty = is_k ? k_empty : v_empty;
    const CUtensorMap *ctx = is_k ? &maps.kx : &maps.vx, *chunk = is_k ? &maps.kc : &maps.vc;
    TileSource* source = reinterpret_cast<TileSource*>(smem + Smem::kSource) + (is_k ? 0 : 1);
    const uint32_t bytes = sparse_tile_bytes<D>(g);
    ListWalker w;
    w.open(g, list, count, lane, first);
    for (int j = 0;; ++j) {
      const int st = j % kDecodeStages;
      uint32_t valid;
      const bool last = next_tile(g, w, h, b, a.cache_shared ? 0 : b, source, valid);   // before the wait for the stage
      if (!mbar_wait_ok(empty + st, ((j / kDecodeStages) & 1) ^ 1, abort_flag)) break;
      if (lane == 0) {
        if (is_k) {   // the readers of the stage's last descriptor have returned its K
          desc[st].valid = valid;
          desc[st].flags = last ? kTileLast : 0u;
        }
        mbar_arrive_expect_tx(full + st, bytes);
        load_sparse_tile<D>(ring + st * TileGeom<D>::kBytes, ctx, chunk, full + st, source, g);
      }
      __syncwarp();
      if (last) break;
    }
  } else {
    // scores: lane = (key of the warp's, part of the head dimension); output: lane = (piece of 8 columns, group of keys)
    constexpr int kLanes = 32 / kKeys, kMine = D / 8 / kLanes;
    constexpr int kPieces = D / 8, kGroups = 32 / kPieces, kPerGroup = kKeys / kGroups;
    const int key = warp * kKeys + lane / kLanes, sub = lane % kLanes;
    const int piece = lane % kPieces, group = lane / kPieces;
    float q[R][kMine][8], m[R], l[R], o[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const __nv_bfloat16* row = a.q + ((static_cast<long long>(b) * R + r) * a.heads + h) * D;
#pragma unroll
      for (int c = 0; c < kMine; ++c)
        unpack8(*reinterpret_cast<const uint4*>(row + score_piece<D>(kLanes, sub, c) * 8), q[r][c]);
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[r][e] = 0.f;
    }
    for (int j = 0;; ++j) {
      const int st = j % kDecodeStages;
      const uint32_t phase = (j / kDecodeStages) & 1;
      bool ok = mbar_wait_ok(k_full + st, phase, abort_flag);
      const uint32_t flags = reinterpret_cast<volatile TileDesc*>(desc + st)->flags;
      const uint32_t valid4 = reinterpret_cast<volatile TileDesc*>(desc + st)->valid;
      const int valid = static_cast<int>((valid4 >> (8 * (warp * kKeys / 32))) & 0xff) - warp * kKeys % 32;   // of this warp's keys
      const uint8_t *k = sK + st * TileGeom<D>::kBytes, *v = sV + st * TileGeom<D>::kBytes;
      float w[R];
      if (valid > 0) {   // the same for the whole warp
        float s[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r][0] = s[r][1] = 0.f;
#pragma unroll
        for (int c = 0; c < kMine; ++c) {
          float f[8];
          unpack8(tile_piece(k, key, score_piece<D>(kLanes, sub, c)), f);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[r][e & 1] = fmaf(q[r][c][e], f[e], s[r][e & 1]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float x = s[r][0] + s[r][1];
#pragma unroll
          for (int step = 1; step < kLanes; step *= 2) x += __shfl_xor_sync(0xffffffffu, x, step);
          x = lane / kLanes < valid ? x * a.scale_log2 : -INFINITY;
          float top = x;
#pragma unroll
          for (int step = kLanes; step < 32; step *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, step));
          top = fmaxf(top, m[r]);
          const float ref = top == -INFINITY ? 0.f : top;     // no key with a finite score so far
          const float alpha = exp2f(m[r] - ref);
          m[r] = top;
          w[r] = exp2f(x - ref);
          l[r] = l[r] * alpha + (sub == 0 ? w[r] : 0.f);       // summed over the lanes at the end
#pragma unroll
          for (int e = 0; e < 8; ++e) o[r][e] *= alpha;
        }
      }
      warp_arrive(k_empty + st, lane);
      ok = mbar_wait_ok(v_full + st, phase, abort_flag) && ok;
      if (valid > 0) {
#pragma unroll
        for (int i = 0; i < kPerGroup; ++i) {
          const int at = group * kPerGroup + i;
          float f[8];
          unpack8(tile_piece(v, warp * kKeys + at, piece), f);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float p = __shfl_sync(0xffffffffu, w[r], at * kLanes);   // 0 behind `valid`, where V's rows are zeros
#pragma unroll
            for (int e = 0; e < 8; ++e) o[r][e] = fmaf(p, f[e], o[r][e]);
          }
        }
      }
      warp_arrive(v_empty + st, lane);
      if ((flags & kTileLast) || !__all_sync(0xffffffffu, ok)) break;
    }
    // the groups of keys of the warp, then what the warp has to say
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int x = 1; x < 32; x *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x);
#pragma unroll
      for (int x = kPieces; x < 32; x *= 2)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[r][e] += __shfl_xor_sync(0xffffffffu, o[r][e], x);
      float* dst = s_out + (warp * R + r) * D + piece * 8;
      if (lane < kPieces) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = o[r][e];
      }
      if (lane == 0) {
        s_stat[(warp * R + r) * 2] = m[r];
        s_stat[(warp * R + r) * 2 + 1] = l[r];
      }
    }
  }
  settle_after_abort(abort_flag);
  __syncthreads();
  // the CTA's warps joined, one thread per column: weights exp2(m - the largest m)
  float* s_joined = reinterpret_cast<float*>(smem + Smem::kJoined);
  for (int i = tid; i < R * D; i += kThreads) {
    const int r = i / D, d = i - r * D;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) top = fmaxf(top, s_stat[(x * R + r) * 2]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f, acc = 0.f;
#pragma unroll
    for (int x = 0; x < kWarps; ++x) {
      const float w = exp2f(s_stat[(x * R + r) * 2] - ref);
      sum = fmaf(w, s_stat[(x * R + r) * 2 + 1], sum);
      acc = fmaf(w, s_out[(x * R + r) * D + d], acc);
    }
    s_out[r * D + d] = acc;   // warp 0's place: nobody else reads this column
    if (d == 0) {
      s_joined[r * 2] = top;
      s_joined[r * 2 + 1] = sum;
    }
  }
  cluster_sync_all();
  if (part == 0) {   // then the CTAs
    for (int i = tid; i < R * D; i += kThreads) {
      const int r = i / D, d = i - r * D;
      float m[kDecodeMaxCluster], l[kDecodeMaxCluster], v[kDecodeMaxCluster], top = -INFINITY;
#pragma unroll
      for (int c = 0; c < kDecodeMaxCluster; ++c) {
        m[c] = -INFINITY;
        l[c] = v[c] = 0.f;
        if (c < parts) {
          m[c] = ld_cluster(cluster_map(smem_u32(s_joined + r * 2), c));
          l[c] = ld_cluster(cluster_map(smem_u32(s_joined + r * 2 + 1), c));
          v[c] = ld_cluster(cluster_map(smem_u32(s_out + r * D + d), c));
        }
      }
#pragma unroll
      for (int c = 0; c < kDecodeMaxCluster; ++c) top = fmaxf(top, m[c]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f, acc = 0.f;
#pragma unroll
      for (int c = 0; c < kDecodeMaxCluster; ++c) {
        const float w = exp2f(m[c] - ref);
        sum = fmaf(w, l[c], sum);
        acc = fmaf(w, v[c], acc);
      }
      a.o[((static_cast<long long>(b) * R + r) * a.heads + h) * D + d] = __float2bfloat16_rn(sum == 0.f ? 0.f : acc / sum);
      if (d == 0 && a.lse != nullptr)
        a.lse[(static_cast<long long>(b) * a.heads + h) * R + r] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
    }
  }
  cluster_sync_all();   // the parts stay in place until they have been read
}

}  // namespace astro
