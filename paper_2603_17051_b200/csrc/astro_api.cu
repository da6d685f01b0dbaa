// C ABI of the rolling-KV chunk-attention library: host-side cache metadata, argument checks,
// tensor-map construction and kernel launches.  Declarations and semantics: include/astro.h.
#include "astro.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>

#include "attn_bwd.cuh"
#include "attn_fwd.cuh"
#include "attn_fwd_pair.cuh"
#include "block_select.cuh"
#include "kv_ring.cuh"
#include "nft_loss.cuh"
#include "rope.cuh"
#include "sparse_bwd.cuh"
#include "sparse_decode.cuh"
#include "sparse_fwd.cuh"

using namespace astro;

struct astro_kvcache {
  astro_kvcache_desc_t d;
  void* k;
  void* v;
  int sink_held;   // frames in sink slots [0, S)
  int win_head;    // ring index (0..L-1) of the oldest window frame
  int win_held;    // frames in the window ring, slots S + (head + i) % L
  int64_t frames_seen;
  // Tensor maps of the storage: built once (by create when a driver is present, else by the first attention
  // call) under a once-flag, read-only afterwards, so attention calls from several threads may share a handle.
  mutable std::once_flag maps_once;
  mutable astro_status_t maps_status;
  mutable CUtensorMap tm_k, tm_v;
};

struct astro_rope {
  astro_rope_desc_t d;
  double frequency[kRopeMaxPairs];
  double magnitude;
  RopeTable table;
};

namespace astro {
// Self-test of the bounded wait: one warp waits on an mbarrier that nothing will ever complete.  The wait
// gives up after `cycle_limit` clocks, records the time-out in the device status word and the kernel ends
// normally, which is exactly the path a broken hand-off in the attention kernels would take.  Only the first lane waits on
// that barrier, the others on one that is complete: every form of the wait has to tell all of them that it failed.
__global__ void wait_timeout_selftest_kernel(long long cycle_limit) {
  __shared__ uint64_t never, done;
  __shared__ int abort_flag;
  if (threadIdx.x == 0) {
    mbar_init(&never, 1);
    mbar_init(&done, 1);
    abort_flag = 0;
    fence_mbar_init();
    mbar_arrive(&done);
  }
  __syncthreads();
  uint64_t* bar = threadIdx.x == 0 ? &never : &done;
  bool went_on = mbar_wait_ok(bar, 0, &abort_flag, cycle_limit);
  went_on = mbar_wait_relaxed_ok(bar, 0, &abort_flag) || went_on;   // these two return at once: the flag is up
  went_on = mbar_wait_at_ok(smem_u32(bar), 0, smem_u32(&abort_flag)) || went_on;
  if (went_on) atomicOr(&g_device_status, kStatusWarpParted);
}
}  // namespace astro

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool desc_ok(const astro_kvcache_desc_t* d) {
  return d && d->cache_batch >= 1 && d->heads >= 1 && (d->head_dim == 64 || d->head_dim == 128) &&
         d->tokens_per_frame >= 1 && d->sink_frames >= 0 && d->window_frames >= 1;
}

// ---- device / driver helpers -------------------------------------------------------------------
// Per-device facts are cached in atomics: several host threads may make their first call at the same time,
// and all of them would store the same value.
constexpr int kMaxDevices = 64;

astro_status_t check_arch() {
  static std::atomic<int> ok_device[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (dev >= 0 && dev < kMaxDevices && ok_device[dev].load(std::memory_order_acquire)) return ASTRO_OK;
  int major = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (major != 10) return ASTRO_ERR_ARCH;
  if (dev >= 0 && dev < kMaxDevices) ok_device[dev].store(1, std::memory_order_release);
  return ASTRO_OK;
}

// Number of SMs of the current device (0 if it cannot be read).
int sm_count() {
  static std::atomic<int> count[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev >= 0 && dev < kMaxDevices) {
    const int c = count[dev].load(std::memory_order_acquire);
    if (c > 0) return c;
  }
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev >= 0 && dev < kMaxDevices) count[dev].store(n, std::memory_order_release);
  return n;
}

typedef CUresult (*encode_tiled_fn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

encode_tiled_fn get_encode_fn() {
  static encode_tiled_fn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<encode_tiled_fn>(p);
  });
  return fn;
}

// bf16 tensor seen as {d, token, head, batch} with byte strides; box = 64 columns x 128 tokens, 128-byte
// swizzle, zero fill outside the tensor.
astro_status_t make_tmap(CUtensorMap* out, const void* base, int head_dim, long long n_tok, int heads, int batch,
                         unsigned long long stride_tok, unsigned long long stride_head,
                         unsigned long long stride_batch, int box_rows = kTile) {
  encode_tiled_fn fn = get_encode_fn();
  if (!fn) return ASTRO_ERR_CUDA;
  cuuint64_t dims[4] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(n_tok),
                        static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(batch)};
  cuuint64_t strides[3] = {stride_tok, stride_head, stride_batch};
  cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  CUresult r = fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ASTRO_OK : ASTRO_ERR_CUDA;
}

// Caller tensor [batch, n_tok, H, D].
astro_status_t make_tmap_user(CUtensorMap* out, const void* base, int head_dim, int n_tok, int heads, int batch,
                              int box_rows = kTile) {
  const unsigned long long row = static_cast<unsigned long long>(head_dim) * 2;
  return make_tmap(out, base, head_dim, n_tok, heads, batch, row * heads, row, row * heads * n_tok, box_rows);
}

// Cache storage seen up to token `end_tok` only (rows from there on read as zeros), box of `box_rows` tokens.
astro_status_t make_tmap_cache_range(CUtensorMap* out, const astro_kvcache* c, const void* base, long long end_tok,
                                     int box_rows) {
  const auto& d = c->d;
  const long long tok = static_cast<long long>(d.sink_frames + d.window_frames) * d.tokens_per_frame;
  const unsigned long long row = static_cast<unsigned long long>(d.head_dim) * 2;
  return make_tmap(out, base, d.head_dim, end_tok, d.heads, d.cache_batch, row, row * tok, row * tok * d.heads,
                   box_rows);
}

astro_status_t build_cache_maps(const astro_kvcache* c) {
  const auto& d = c->d;
  const long long tok = static_cast<long long>(d.sink_frames + d.window_frames) * d.tokens_per_frame;
  const unsigned long long row = static_cast<unsigned long long>(d.head_dim) * 2;
  astro_status_t s = make_tmap(&c->tm_k, c->k, d.head_dim, tok, d.heads, d.cache_batch, row, row * tok,
                               row * tok * d.heads);
  if (s != ASTRO_OK) return s;
  s = make_tmap(&c->tm_v, c->v, d.head_dim, tok, d.heads, d.cache_batch, row, row * tok, row * tok * d.heads);
  return s;
}

astro_status_t cache_maps(const astro_kvcache* c) {
  std::call_once(c->maps_once, [c] { c->maps_status = build_cache_maps(c); });
  return c->maps_status;
}

// Physical token ranges of the held frames, merged where adjacent, followed by the chunk's keys.
KeySegs build_segments(const astro_kvcache* c, int n_kc) {
  KeySegs s;
  std::memset(&s, 0, sizeof(s));
  auto push = [&s](long long start, long long count, int from_chunk) {
    if (count <= 0) return;
    if (s.n > 0 && !from_chunk && !s.from_chunk[s.n - 1] && s.start[s.n - 1] + s.count[s.n - 1] == start) {
      s.count[s.n - 1] += static_cast<int>(count);
      return;
    }
    s.start[s.n] = static_cast<int>(start);
    s.count[s.n] = static_cast<int>(count);
    s.from_chunk[s.n] = from_chunk;
    ++s.n;
  };
  if (c) {
    const int T = c->d.tokens_per_frame, S = c->d.sink_frames, L = c->d.window_frames;
    const int first = c->win_held < L - c->win_head ? c->win_held : L - c->win_head;  // frames before the wrap
    const int wrapped = c->win_held - first;
    push(0, static_cast<long long>(c->sink_held) * T, 0);
    push(static_cast<long long>(S) * T, static_cast<long long>(wrapped) * T, 0);
    push(static_cast<long long>(S + c->win_head) * T, static_cast<long long>(first) * T, 0);
  }
  push(0, n_kc, 1);
  return s;
}

template <typename K> astro_status_t set_smem(K kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess
             ? ASTRO_OK
             : ASTRO_ERR_CUDA;
}

template <typename K> astro_status_t set_smem_once(K kernel, int bytes, std::atomic<int> (&done)[kMaxDevices]) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (dev >= 0 && dev < kMaxDevices && done[dev].load(std::memory_order_acquire)) return ASTRO_OK;
  astro_status_t s = set_smem(kernel, bytes);   // idempotent: a second thread repeating it does no harm
  if (s == ASTRO_OK && dev >= 0 && dev < kMaxDevices) done[dev].store(1, std::memory_order_release);
  return s;
}

astro_status_t launch_status() { return cudaGetLastError() == cudaSuccess ? ASTRO_OK : ASTRO_ERR_CUDA; }

// Launches a kernel as the dependent of the one launched just before it on the stream: it may start while that one
// drains, and waits for it itself (dependency_wait).
template <typename... Params, typename... Args>
astro_status_t launch_dependent(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) == cudaSuccess ? launch_status() : ASTRO_ERR_CUDA;
}

struct AttnArgs {
  const astro_kvcache* cache;
  int batch, heads, head_dim, n_q, n_kc;
};

astro_status_t check_attn_args(const AttnArgs& a, float scale) {
  if (a.batch < 1 || a.heads < 1 || a.n_q < 1 || a.n_kc < 0) return ASTRO_ERR_SHAPE;
  if (a.head_dim != 64 && a.head_dim != 128) return ASTRO_ERR_SHAPE;
  if (!(scale >= 0.f) || !(scale < 3.0e38f)) return ASTRO_ERR_SHAPE;
  if (a.batch > 65535 || a.heads > 65535) return ASTRO_ERR_SHAPE;
  int held = 0;
  if (a.cache) {
    const auto& d = a.cache->d;
    if (d.heads != a.heads || d.head_dim != a.head_dim) return ASTRO_ERR_SHAPE;
    if (d.cache_batch != a.batch && d.cache_batch != 1) return ASTRO_ERR_SHAPE;
    held = a.cache->sink_held + a.cache->win_held;
  }
  if (held == 0 && a.n_kc == 0) return ASTRO_ERR_SHAPE;  // no key at all: softmax undefined
  return ASTRO_OK;
}

// 0: fast pass with the safe pass as fallback (normal operation); 1: safe pass only; 2: CTA-pair kernel where the
// shape allows it (head_dim 128).  Diagnostics and tests.
std::atomic<int> g_fwd_mode{0};

// Set by the CTA-pair kernel when a row needs the running-reference pass; read back by astro_debug_pair_flag.
__device__ int g_pair_needs_safe = 0;

astro_status_t launch_fwd_pair(const AttnArgs& a, const astro_kvcache* cache, bool have_ctx, const void* q,
                               const void* k_chunk, const void* v_chunk, const KeySegs& segs, float scale, void* o,
                               float* lse, cudaStream_t st) {
  static std::atomic<int> done[kMaxDevices];
  astro_status_t s = set_smem_once(chunk_attn_fwd_pair_kernel, PairSmem::kTotal, done);
  if (s != ASTRO_OK) return s;
  PairMaps maps;
  std::memset(&maps, 0, sizeof(maps));
  if (a.n_kc > 0) {
    if ((s = make_tmap_user(&maps.kc, k_chunk, 128, a.n_kc, a.heads, a.batch, 64)) != ASTRO_OK) return s;
    if ((s = make_tmap_user(&maps.vc, v_chunk, 128, a.n_kc, a.heads, a.batch)) != ASTRO_OK) return s;
  }
  if (have_ctx) {
    int ci = 0;
    for (int i = 0; i < segs.n; ++i) {
      if (segs.from_chunk[i]) continue;
      const long long end = static_cast<long long>(segs.start[i]) + segs.count[i];
      if ((s = make_tmap_cache_range(&maps.kx[ci], cache, cache->k, end, 64)) != ASTRO_OK) return s;
      if ((s = make_tmap_cache_range(&maps.vx[ci], cache, cache->v, end, kTile)) != ASTRO_OK) return s;
      ++ci;
    }
  }
  int* flag = nullptr;
  if (cudaGetSymbolAddress(reinterpret_cast<void**>(&flag), g_pair_needs_safe) != cudaSuccess) return ASTRO_ERR_CUDA;
  const int shared = (cache && cache->d.cache_batch == 1 && a.batch > 1) ? 1 : 0;
  const int tiles = (a.n_q + kTile - 1) / kTile;
  dim3 grid((tiles + 1) / 2 * 2, shared ? a.batch : a.heads, shared ? a.heads : a.batch);
  chunk_attn_fwd_pair_kernel<<<grid, kPairThreads, PairSmem::kTotal, st>>>(
      static_cast<const __nv_bfloat16*>(q), maps, segs, a.n_q, a.heads, shared, scale * kLog2e,
      static_cast<__nv_bfloat16*>(o), lse, flag);
  return launch_status();
}

template <int D>
astro_status_t launch_fwd(const AttnArgs& a, const __nv_bfloat16* q, const CUtensorMap& tkc, const CUtensorMap& tvc,
                          const CUtensorMap& tkx, const CUtensorMap (&tvx)[2], const KeySegs& segs, float scale,
                          void* o, float* lse, cudaStream_t st) {
  static std::atomic<int> done[kMaxDevices];
  astro_status_t s = set_smem_once(chunk_attn_fwd_kernel<D>, FwdSmem<D>::kTotal, done);
  if (s != ASTRO_OK) return s;
  const int shared = (a.cache && a.cache->d.cache_batch == 1 && a.batch > 1) ? 1 : 0;
  // One CTA per SM, each walking over its share of the (query tile, head, sample) units; more CTAs only when a
  // CTA would get more units than it has redo bits for.
  const long long units = static_cast<long long>((a.n_q + kTile - 1) / kTile) * a.heads * a.batch;
  const int sms = sm_count();
  if (sms <= 0) return ASTRO_ERR_CUDA;
  if (units > 0x7fffffffLL) return ASTRO_ERR_SHAPE;
  long long ctas = units < sms ? units : sms;
  if (units > ctas * kFwdMaxUnits) ctas = sms * ((units + static_cast<long long>(sms) * kFwdMaxUnits - 1) / (static_cast<long long>(sms) * kFwdMaxUnits));
  chunk_attn_fwd_kernel<D><<<static_cast<unsigned>(ctas), kFwdThreads, FwdSmem<D>::kTotal, st>>>(
      q, tkc, tvc, tkx, tvx[0], tvx[1], segs, a.batch, a.n_q, a.heads, shared,
      scale * kLog2e, g_fwd_mode.load(std::memory_order_relaxed) == 1 ? 1 : 0, static_cast<__nv_bfloat16*>(o), lse);
  return launch_status();
}

template <int D>
astro_status_t launch_bwd_delta(const void* o, const void* d_o, int batch, int heads, int n_q, float* delta,
                                cudaStream_t st) {
  const long long rows = static_cast<long long>(batch) * n_q * heads;
  const unsigned blocks = static_cast<unsigned>((rows * 32 + 255) / 256);
  bwd_delta_kernel<D><<<blocks, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(o),
                                             static_cast<const __nv_bfloat16*>(d_o), delta, batch, n_q, heads);
  return launch_status();
}

template <int D>
astro_status_t launch_bwd_dq(const AttnArgs& a, const __nv_bfloat16* q, const CUtensorMap& tdo, const CUtensorMap& tkc,
                             const CUtensorMap& tvc, const CUtensorMap (&tkx)[2], const CUtensorMap& tvx,
                             const KeySegs& segs, float scale, const float* lse, const float* delta, void* dq,
                             cudaStream_t st) {
  static std::atomic<int> done[kMaxDevices];
  astro_status_t s = set_smem_once(chunk_attn_bwd_dq_kernel<D>, DqSmem<D>::kTotal, done);
  if (s != ASTRO_OK) return s;
  const int shared = (a.cache && a.cache->d.cache_batch == 1 && a.batch > 1) ? 1 : 0;
  dim3 grid_q((a.n_q + kTile - 1) / kTile, shared ? a.batch : a.heads, shared ? a.heads : a.batch);
  chunk_attn_bwd_dq_kernel<D><<<grid_q, kDqThreads, DqSmem<D>::kTotal, st>>>(
      q, tdo, tkc, tvc, tkx[0], tkx[1], tvx, segs, a.n_q, a.heads, shared, scale, lse, delta,
      static_cast<__nv_bfloat16*>(dq));
  return launch_status();
}

template <int D>
astro_status_t launch_bwd_dkv(const AttnArgs& a, const CUtensorMap& tq, const CUtensorMap& tdo,
                              const CUtensorMap& tkc, const CUtensorMap& tvc, float scale, const float* lse,
                              const float* delta, void* dk, void* dv, cudaStream_t st) {
  static std::atomic<int> done[kMaxDevices];
  astro_status_t s = set_smem_once(chunk_attn_bwd_dkv_kernel<D>, DkvSmem<D>::kTotal, done);
  if (s != ASTRO_OK) return s;
  dim3 grid_k((a.n_kc + kTile - 1) / kTile, a.heads, a.batch);
  chunk_attn_bwd_dkv_kernel<D><<<grid_k, kDkvThreads, DkvSmem<D>::kTotal, st>>>(
      tq, tdo, tkc, tvc, a.n_q, a.n_kc, a.heads, scale, lse, delta, static_cast<__nv_bfloat16*>(dk),
      static_cast<__nv_bfloat16*>(dv));
  return launch_status();
}

// Copies frames between a caller tensor and the storage slots listed in `slots` (logical order).
template <bool ToCache>
astro_status_t launch_ring_copy(const astro_kvcache* c, void* k_user, void* v_user, const int* slots, int n_frames,
                                cudaStream_t st) {
  const auto& d = c->d;
  const int vpr = d.head_dim * 2 / 16;
  const int row_vecs = d.heads * vpr;
  const int threads = row_vecs >= 256 ? 256 : ((row_vecs + 31) / 32) * 32;
  const int chunks_per_frame = (d.tokens_per_frame + kRingTokensPerThread - 1) / kRingTokensPerThread;
  if (d.cache_batch > 32767 || static_cast<long long>(chunks_per_frame) * kMaxFramesPerCopy > 65535)
    return ASTRO_ERR_SHAPE;
  for (int f0 = 0; f0 < n_frames; f0 += kMaxFramesPerCopy) {
    SlotMap map;
    map.n = n_frames - f0 < kMaxFramesPerCopy ? n_frames - f0 : kMaxFramesPerCopy;
    for (int j = 0; j < map.n; ++j) map.slot[j] = slots[f0 + j];
    dim3 grid((row_vecs + threads - 1) / threads, map.n * chunks_per_frame, 2 * d.cache_batch);
    ring_copy_kernel<ToCache><<<grid, threads, 0, st>>>(
        static_cast<uint4*>(k_user), static_cast<uint4*>(v_user), static_cast<uint4*>(c->k),
        static_cast<uint4*>(c->v), map, d.heads, d.tokens_per_frame, vpr, d.sink_frames + d.window_frames, f0,
        n_frames, chunks_per_frame);
  }
  return launch_status();
}

// Whether a tensor of these sizes and strides (elements) with contiguous rows of `row` elements overlaps itself.
bool overlaps_itself(const long long (&size)[3], const long long (&stride)[3], long long row) {
  int order[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[order[j]] < stride[order[i]]) { const int x = order[i]; order[i] = order[j]; order[j] = x; }
  long long span = row;
  for (int i = 0; i < 3; ++i) {
    if (size[order[i]] <= 1) continue;
    if (stride[order[i]] < span) return true;
    span += stride[order[i]] * (size[order[i]] - 1);
  }
  return false;
}

template <typename T, int MODE>
astro_status_t launch_rope(const astro_rope* rope, const RopeTensors& x, const int* positions, int per_sample, int n_tokens,
                           int total_tokens, float sign, cudaStream_t st) {
  const int per_row = rope_items_per_row(MODE, rope->d.head_dim, rope->d.rot_dim, RopeVec<T>::kElems);
  const int rows = x.heads_q + x.heads_k, sms = sm_count();
  if (sms <= 0) return ASTRO_ERR_CUDA;
  // as many row phases as bring every SM about 512 threads, each phase with a row at least (chunk of 4680
  // tokens: 12.1 us, with 1024 threads 15.7, more angles and a second wave of blocks)
  const long long threads = static_cast<long long>(total_tokens) * per_row;
  long long phases = (sms * 512ll + threads - 1) / threads;
  if (phases > rows) phases = rows;
  const long long blocks = (threads * phases + kRopeThreads - 1) / kRopeThreads;
  if (blocks > 0x7fffffffLL) return ASTRO_ERR_SHAPE;
  rope_kernel<T, MODE><<<static_cast<unsigned>(blocks), kRopeThreads, 0, st>>>(
      rope->table, x, positions, per_sample, n_tokens, total_tokens, rope->d.head_dim, rope->d.rot_dim, static_cast<int>(phases), sign);
  return launch_status();
}

template <typename T>
astro_status_t launch_rope_typed(const astro_rope* rope, const RopeTensors& x, const int* positions, int per_sample,
                                 int n_tokens, int total_tokens, float sign, cudaStream_t st) {
  if (rope->d.layout == ASTRO_ROPE_INTERLEAVED)
    return launch_rope<T, kRopeInterleaved>(rope, x, positions, per_sample, n_tokens, total_tokens, sign, st);
  if (rope->d.rot_dim / 2 % RopeVec<T>::kElems == 0)
    return launch_rope<T, kRopeHalves>(rope, x, positions, per_sample, n_tokens, total_tokens, sign, st);
  return launch_rope<T, kRopeHalvesScalar>(rope, x, positions, per_sample, n_tokens, total_tokens, sign, st);
}

bool block_tokens_ok(int block) { return block >= 8 && block <= kTile && block % 8 == 0; }

// The key blocks of a call (block size and counts already checked); false if their number does not fit an int.
bool build_key_blocks(const astro_kvcache* c, int n_kc, int block, KeyBlocks* out) {
  KeyBlocks kb;
  std::memset(&kb, 0, sizeof(kb));
  kb.block = block;
  kb.n_kc = n_kc;
  long long ctx = 0;
  kb.per_frame = kb.tokens_per_frame = kb.win_slots = 1;
  if (c) {
    kb.tokens_per_frame = c->d.tokens_per_frame;
    kb.per_frame = (kb.tokens_per_frame - 1) / block + 1;
    kb.sink_held = c->sink_held;
    kb.sink_slots = c->d.sink_frames;
    kb.win_head = c->win_head;
    kb.win_slots = c->d.window_frames;
    ctx = static_cast<long long>(c->sink_held + c->win_held) * kb.per_frame;
  }
  const long long total = ctx + (static_cast<long long>(n_kc) + block - 1) / block;
  if (total > 0x3fffffffLL) return false;
  kb.ctx = static_cast<int>(ctx);
  kb.total = static_cast<int>(total);
  *out = kb;
  return true;
}

// As many warps per block of tokens as bring the GPU about 1500 of them, so that enough loads are in flight (1872
// blocks: one warp each 15.5 us, two 17.9: more streams, more sums to join).
int pool_share(long long blocks) {
  int share = 1;
  while (share < 8 && blocks * share < 1500) share *= 2;
  return share;
}

template <int D>
astro_status_t launch_pool(const PoolSource& s, int heads, int batch, const KeyBlocks& kb, int frame0, cudaStream_t st) {
  const int share = pool_share(static_cast<long long>(s.blocks) * heads * batch), per_cta = kPoolThreads / 32 / share;
  dim3 grid((s.blocks + per_cta - 1) / per_cta, heads, batch);
  block_pool_kernel<D><<<grid, kPoolThreads, 0, st>>>(s, kb, frame0, share);
  return launch_status();
}

void set_inverses(PoolSource* s) {
  const int rest = s->tokens % s->block;
  s->inv_block = 1.0 / s->block;
  s->inv_last = 1.0 / (rest ? rest : s->block);
}

template <int D>
astro_status_t launch_select(const PoolSource& q, const PoolSource& kc, SelectArgs a, const KeyBlocks& kb, int batch,
                             cudaStream_t st) {
  static std::atomic<int> done[kMaxDevices];
  astro_status_t s = set_smem_once(block_select_kernel<D>, ASTRO_SELECT_MAX_BLOCKS * 8, done);
  if (s != ASTRO_OK) return s;
  const long long units = static_cast<long long>(q.blocks) + kc.blocks;
  const bool fused = units <= kSelectWarps;   // a warp for every mean (both sides measured: see the kernel)
  // thread blocks of a head: a tile's eight query blocks each, or as many as have room for their keys in shared memory
  const int room = ASTRO_SELECT_MAX_BLOCKS / kb.total;
  a.rows = room < kSelectRows ? room : kSelectRows;
  int size = (a.q_blocks + a.rows - 1) / a.rows;
  if (!fused) {
    // four warps per thread block where that is enough: spreads 912 means better over the SMs (21.9 us against 22.5 in all)
    const int share = pool_share(units * a.heads * batch), warps = share > 4 ? share : 4, per_cta = warps / share;
    dim3 grid(static_cast<unsigned>((units + per_cta - 1) / per_cta), a.heads, batch);
    block_mean_kernel<D><<<grid, 32 * warps, 0, st>>>(q, kc, share);
    if ((s = launch_status()) != ASTRO_OK) return s;
    return launch_dependent(block_select_kernel<D>, dim3(size, a.heads, batch), kSelectThreads,
                            static_cast<size_t>(a.rows) * kb.total * 8, st, a, kb, q, kc, 0);
  }
  if (size > 8) size = 8;
  int share = 1;
  while (units * share * 2 <= kSelectWarps) share *= 2;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = static_cast<unsigned>(size);
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(size), a.heads, batch);
  cfg.blockDim = dim3(kSelectThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(a.rows) * kb.total * 8;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, block_select_kernel<D>, a, kb, q, kc, share) == cudaSuccess ? launch_status() : ASTRO_ERR_CUDA;
}

// ---- attention over lists of key blocks ---------------------------------------------------------------------
// bf16 tensor seen as {d, token, slot, head, batch}: rows from `tokens` on read as zeros in every slot.
astro_status_t make_tmap5(CUtensorMap* out, const void* base, int head_dim, long long tokens, int slots, int heads, int batch,
                          unsigned long long st_tok, unsigned long long st_slot, unsigned long long st_head,
                          unsigned long long st_batch, int box_rows) {
  encode_tiled_fn fn = get_encode_fn();
  if (!fn) return ASTRO_ERR_CUDA;
  cuuint64_t dims[5] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(tokens), static_cast<cuuint64_t>(slots),
                        static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(batch)};
  cuuint64_t strides[4] = {st_tok, st_slot, st_head, st_batch};
  cuuint32_t box[5] = {64, static_cast<cuuint32_t>(box_rows), 1, 1, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  CUresult r = fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? ASTRO_OK : ASTRO_ERR_CUDA;
}

struct SparseCall {
  AttnArgs a;
  const void *q, *k_chunk, *v_chunk;
  const int32_t* blocks;
  int n_select, block_tokens;
};

astro_status_t check_sparse(const SparseCall& c, float scale, SparseGeom* g) {
  astro_status_t s = check_attn_args(c.a, scale);
  if (s != ASTRO_OK) return s;
  if (!block_tokens_ok(c.block_tokens) || c.n_select < 1 || c.n_select > ASTRO_MAX_SELECT ||
      !build_key_blocks(c.a.cache, c.a.n_kc, c.block_tokens, &g->kb))
    return ASTRO_ERR_SHAPE;
  g->pad = sparse_pad(c.block_tokens);
  g->per_tile = kTile / g->pad;
  g->chunk_fill = g->kb.ctx == 0 ? 1 : 0;
  return ASTRO_OK;
}

astro_status_t sparse_maps(const SparseCall& c, const SparseGeom& g, SparseMaps* m) {
  std::memset(m, 0, sizeof(*m));
  astro_status_t s = ASTRO_OK;
  const unsigned long long row = static_cast<unsigned long long>(c.a.head_dim) * 2;
  if (c.a.n_kc > 0) {
    const unsigned long long all = row * c.a.heads * c.a.n_kc;
    for (int i = 0; i < 2 && s == ASTRO_OK; ++i)
      s = make_tmap5(i ? &m->vc : &m->kc, i ? c.v_chunk : c.k_chunk, c.a.head_dim, c.a.n_kc, 1, c.a.heads, c.a.batch,
                     row * c.a.heads, all, row, all, g.kb.block);
  }
  if (g.kb.ctx > 0 && s == ASTRO_OK) {
    const auto& d = c.a.cache->d;
    const int slots = d.sink_frames + d.window_frames;
    const unsigned long long frame = row * d.tokens_per_frame;
    for (int i = 0; i < 2 && s == ASTRO_OK; ++i)
      s = make_tmap5(i ? &m->vx : &m->kx, i ? c.a.cache->v : c.a.cache->k, d.head_dim, d.tokens_per_frame, slots, d.heads,
                     d.cache_batch, row, frame, frame * slots, frame * slots * d.heads, g.kb.block);
  }
  return s;
}

// Into how many ranges a unit's list is cut, and how many entries a range has.  With fewer units than half the SMs of a B200
// (148) most of it would idle while a few CTAs walk over long lists.  Joining the parts costs about 4 us, a tile about 0.7: lists
// of 12 tiles and more are cut, into ranges of 4 tiles and more.
struct SparseSplit {
  int splits, entries;
};
SparseSplit sparse_split(int batch, int heads, int n_q, int n_select, int block_tokens) {
  constexpr int kSms = 148;
  const long long units = static_cast<long long>((n_q - 1) / kTile + 1) * heads * batch;
  const int per_tile = kTile / sparse_pad(block_tokens);
  const int tiles = (n_select - 1) / per_tile + 1;
  SparseSplit r{1, n_select};
  if (n_q <= kDecodeMaxQueries || units * 2 > kSms || tiles < 12) return r;   // one or two queries: a kernel of their own
  int want = static_cast<int>(kSms / units);
  if (want > tiles / 4) want = tiles / 4;
  const int each = (tiles - 1) / want + 1;   // tiles of a range
  r.splits = (tiles - 1) / each + 1;
  r.entries = each * per_tile;
  return r;
}

// One or two queries per sample: a cluster of CTAs per list (3 and more queries go to the MMA kernel: every query costs this
// one as much arithmetic as the first).  Clusters do not straddle the GPU's processing clusters, so fewer fit than the
// number of SMs says (48 of three CTAs do not): the size is chosen from what the runtime says fits at a time, to need the
// least rounds * (tiles of a CTA + 8, a CTA's start and end being worth about 8 tiles).
template <int D, int R>
astro_status_t launch_sparse_decode(const SparseCall& c, const SparseGeom& g, float scale, void* o, float* lse, cudaStream_t st) {
  SparseMaps maps;
  astro_status_t s = sparse_maps(c, g, &maps);
  if (s != ASTRO_OK) return s;
  static std::atomic<int> done[kMaxDevices];
  constexpr int kSmem = DecodeSmem<D, R>::kTotal, kThreads = DecodeShape<R>::kThreads;
  if ((s = set_smem_once(sparse_decode_kernel<D, R>, kSmem, done)) != ASTRO_OK) return s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  static std::atomic<int> fits[kMaxDevices][kDecodeMaxCluster + 1];   // clusters of a size at a time, + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return ASTRO_ERR_CUDA;
  const long long lists = static_cast<long long>(c.a.batch) * c.a.heads;
  const int tiles = (c.n_select - 1) / g.per_tile + 1;
  int parts = 1;
  long long least = 0;
  for (int p = 1; p <= kDecodeMaxCluster && p <= tiles; ++p) {
    int n = fits[dev][p].load(std::memory_order_acquire) - 1;
    if (n < 0) {
      attr.val.clusterDim.x = p;
      cfg.gridDim = dim3(p, 1, 1);
      if (cudaOccupancyMaxActiveClusters(&n, sparse_decode_kernel<D, R>, &cfg) != cudaSuccess) {
        (void)cudaGetLastError();
        n = 0;
      }
      fits[dev][p].store(n + 1, std::memory_order_release);
    }
    if (n < 1) continue;
    const long long cost = ((lists + n - 1) / n) * ((tiles + p - 1) / p + 8);
    if (p == 1 || cost < least) { parts = p; least = cost; }
  }
  DecodeArgs a;
  a.q = static_cast<const __nv_bfloat16*>(c.q);
  a.blocks = c.blocks;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.heads = c.a.heads;
  a.n_select = c.n_select;
  a.entries = (tiles + parts - 1) / parts * g.per_tile;
  a.cache_shared = (c.a.cache && c.a.cache->d.cache_batch == 1 && c.a.batch > 1) ? 1 : 0;
  a.scale_log2 = scale * kLog2e;
  attr.val.clusterDim.x = static_cast<unsigned>(parts);
  cfg.gridDim = dim3(static_cast<unsigned>(parts), c.a.heads, c.a.batch);
  return cudaLaunchKernelEx(&cfg, sparse_decode_kernel<D, R>, maps, a, g) == cudaSuccess ? launch_status() : ASTRO_ERR_CUDA;
}

template <int D>
astro_status_t launch_sparse_fwd(const SparseCall& c, const SparseGeom& g, float scale, void* o, float* lse, void* workspace,
                                 cudaStream_t st) {
  const bool careful = g_fwd_mode.load(std::memory_order_relaxed) == 1;   // reaches the MMA kernel's careful pass
  if (c.a.n_q == 1 && !careful) return launch_sparse_decode<D, 1>(c, g, scale, o, lse, st);
  if (c.a.n_q == 2 && !careful) return launch_sparse_decode<D, 2>(c, g, scale, o, lse, st);
  SparseMaps maps;
  astro_status_t s = sparse_maps(c, g, &maps);
  if (s != ASTRO_OK) return s;
  static std::atomic<int> done[kMaxDevices];
  if ((s = set_smem_once(sparse_attn_fwd_kernel<D>, SparseFwdSmem<D>::kTotal, done)) != ASTRO_OK) return s;
  const SparseSplit split = sparse_split(c.a.batch, c.a.heads, c.a.n_q, c.n_select, c.block_tokens);
  const long long rows = static_cast<long long>(c.a.batch) * c.a.heads * c.a.n_q;
  SparseFwdArgs a;
  a.q = static_cast<const __nv_bfloat16*>(c.q);
  a.blocks = c.blocks;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = a.part_o + (split.splits > 1 ? split.splits * rows * D : 0);
  a.batch = c.a.batch; a.heads = c.a.heads; a.n_q = c.a.n_q;
  a.scale_log2 = scale * kLog2e;
  a.careful = careful ? 1 : 0;
  SparseUnits u;
  u.q_tiles = (c.a.n_q - 1) / kTile + 1;
  u.cache_shared = (c.a.cache && c.a.cache->d.cache_batch == 1 && c.a.batch > 1) ? 1 : 0;
  u.dim_y = u.cache_shared ? c.a.batch : c.a.heads;
  u.splits = split.splits;
  u.entries = split.entries;
  u.n_select = c.n_select;
  u.first = 0; u.stride = 0;
  const long long units = static_cast<long long>(u.q_tiles) * c.a.heads * c.a.batch * split.splits;
  const int sms = sm_count();
  if (sms <= 0) return ASTRO_ERR_CUDA;
  if (units > 0x3fffffffLL) return ASTRO_ERR_SHAPE;
  u.total = static_cast<int>(units);
  long long ctas = units < sms ? units : sms;
  if (units > ctas * kFwdMaxUnits) ctas = sms * ((units + static_cast<long long>(sms) * kFwdMaxUnits - 1) / (static_cast<long long>(sms) * kFwdMaxUnits));
  sparse_attn_fwd_kernel<D><<<static_cast<unsigned>(ctas), kSparseThreads, SparseFwdSmem<D>::kTotal, st>>>(maps, a, g, u);
  if ((s = launch_status()) != ASTRO_OK || split.splits == 1) return s;
  return launch_dependent(sparse_combine_kernel<D>, dim3(static_cast<unsigned>((rows + 7) / 8)), 256, 0, st, a.part_o, a.part_lse,
                          split.splits, rows, c.a.n_q, c.a.heads, a.o, lse);
}

// Scratch of the backward: delta, then how often every query tile names every chunk block.
struct SparseBwdScratch {
  size_t delta, counts;   // bytes
};
SparseBwdScratch sparse_bwd_scratch(int batch, int heads, int n_q, int n_kc, int block_tokens) {
  const size_t q_tiles = (n_q - 1) / kTile + 1, blocks = (static_cast<size_t>(n_kc) + block_tokens - 1) / block_tokens;
  SparseBwdScratch s;
  s.delta = (static_cast<size_t>(batch) * heads * n_q * sizeof(float) + 255) & ~static_cast<size_t>(255);
  s.counts = static_cast<size_t>(batch) * heads * blocks * q_tiles * sizeof(int);
  return s;
}

template <int D>
astro_status_t launch_sparse_bwd(const SparseCall& c, const SparseGeom& g, float scale, const void* o, const float* lse,
                                 const void* d_o, void* dq, void* dk, void* dv, void* workspace, cudaStream_t st) {
  SparseMaps maps;
  astro_status_t s = sparse_maps(c, g, &maps);
  if (s != ASTRO_OK) return s;
  CUtensorMap tq, tdo;
  if ((s = make_tmap_user(&tq, c.q, D, c.a.n_q, c.a.heads, c.a.batch)) != ASTRO_OK) return s;
  if ((s = make_tmap_user(&tdo, d_o, D, c.a.n_q, c.a.heads, c.a.batch)) != ASTRO_OK) return s;
  static std::atomic<int> done[kMaxDevices];
  if ((s = set_smem_once(sparse_attn_bwd_kernel<D>, sparse_bwd_smem<D>(), done)) != ASTRO_OK) return s;
  const SparseBwdScratch need = sparse_bwd_scratch(c.a.batch, c.a.heads, c.a.n_q, c.a.n_kc, c.block_tokens);
  float* delta = static_cast<float*>(workspace);
  int* counts = reinterpret_cast<int*>(static_cast<char*>(workspace) + need.delta);
  const int q_tiles = (c.a.n_q - 1) / kTile + 1, chunk_blocks = g.kb.total - g.kb.ctx;
  SparsePrepArgs p;
  p.o = static_cast<const __nv_bfloat16*>(o);
  p.d_o = static_cast<const __nv_bfloat16*>(d_o);
  p.blocks = c.blocks;
  p.delta = delta;
  p.counts = counts;
  p.rows = static_cast<long long>(c.a.batch) * c.a.n_q * c.a.heads;
  p.lists = static_cast<long long>(c.a.batch) * c.a.heads * q_tiles;
  p.heads = c.a.heads; p.n_q = c.a.n_q;
  p.q_tiles = q_tiles;
  p.n_select = c.n_select;
  p.ctx_blocks = g.kb.ctx;
  p.chunk_blocks = chunk_blocks;
  p.spans = (chunk_blocks + kCountSpan - 1) / kCountSpan;
  p.count_blocks = (p.lists * p.spans + kPrepThreads / 32 - 1) / (kPrepThreads / 32);
  const long long per_block = static_cast<long long>(kPrepThreads) * 8 / D * kDeltaRows;
  const long long prep_blocks = p.count_blocks + (p.rows + per_block - 1) / per_block;
  const long long heads = static_cast<long long>(c.a.batch) * c.a.heads, ctas = heads * (q_tiles + chunk_blocks);
  if (prep_blocks > 0x7fffffffLL || ctas > 0x7fffffffLL) return ASTRO_ERR_SHAPE;
  sparse_bwd_prep_kernel<D><<<static_cast<unsigned>(prep_blocks), kPrepThreads, 0, st>>>(p);
  if ((s = launch_status()) != ASTRO_OK) return s;
  SparseBwdArgs a;
  a.q = static_cast<const __nv_bfloat16*>(c.q);
  a.blocks = c.blocks;
  a.lse = lse;
  a.delta = delta;
  a.dq = static_cast<__nv_bfloat16*>(dq);
  a.batch = c.a.batch; a.heads = c.a.heads; a.n_q = c.a.n_q;
  a.q_tiles = q_tiles;
  a.n_select = c.n_select;
  a.cache_shared = (c.a.cache && c.a.cache->d.cache_batch == 1 && c.a.batch > 1) ? 1 : 0;
  a.scale = scale;
  SparseDkvArgs k;
  k.counts = counts;
  k.lse = lse;
  k.delta = delta;
  k.heads = c.a.heads; k.n_q = c.a.n_q; k.n_kc = c.a.n_kc;
  k.q_tiles = q_tiles;
  k.block = c.block_tokens;
  k.chunk_blocks = chunk_blocks;
  k.scale = scale;
  k.dk = static_cast<__nv_bfloat16*>(dk);
  k.dv = static_cast<__nv_bfloat16*>(dv);
  return launch_dependent(sparse_attn_bwd_kernel<D>, dim3(static_cast<unsigned>(ctas)), kSparseBwdThreads, sparse_bwd_smem<D>(), st,
                          maps, tq, tdo, g, a, k, static_cast<int>(heads * q_tiles));
}

}  // namespace

extern "C" {

size_t astro_kvcache_storage_bytes(const astro_kvcache_desc_t* d) {
  if (!desc_ok(d)) return 0;
  return static_cast<size_t>(d->cache_batch) * d->heads * (d->sink_frames + d->window_frames) *
         d->tokens_per_frame * d->head_dim * 2;
}

astro_status_t astro_kvcache_create(const astro_kvcache_desc_t* desc, void* k_storage, void* v_storage,
                                    size_t bytes_each, astro_kvcache_t** out) {
  if (!desc || !k_storage || !v_storage || !out) return ASTRO_ERR_NULL;
  if (!desc_ok(desc)) return ASTRO_ERR_SHAPE;
  if (!aligned16(k_storage) || !aligned16(v_storage)) return ASTRO_ERR_ALIGN;
  if (bytes_each < astro_kvcache_storage_bytes(desc)) return ASTRO_ERR_CAPACITY;
  const long long tok = static_cast<long long>(desc->sink_frames + desc->window_frames) * desc->tokens_per_frame;
  if (tok >= (1ll << 31) - kTile) return ASTRO_ERR_SHAPE;
  astro_kvcache* c = new (std::nothrow) astro_kvcache();
  if (!c) return ASTRO_ERR_CUDA;
  c->d = *desc;
  c->k = k_storage;
  c->v = v_storage;
  c->sink_held = c->win_head = c->win_held = 0;
  c->frames_seen = 0;
  c->maps_status = ASTRO_ERR_CUDA;
  if (get_encode_fn() != nullptr) {   // a driver is present: build the maps now, so attention calls only read them
    const astro_status_t ms = cache_maps(c);
    if (ms != ASTRO_OK) { delete c; return ms; }
  }
  *out = c;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_destroy(astro_kvcache_t* cache) {
  if (!cache) return ASTRO_ERR_NULL;
  delete cache;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_reset(astro_kvcache_t* c) {
  if (!c) return ASTRO_ERR_NULL;
  c->sink_held = c->win_head = c->win_held = 0;
  c->frames_seen = 0;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_append(astro_kvcache_t* c, const void* k, const void* v, int n_frames, void* stream) {
  if (!c || !k || !v) return ASTRO_ERR_NULL;
  if (n_frames < 0) return ASTRO_ERR_SHAPE;
  if (!aligned16(k) || !aligned16(v)) return ASTRO_ERR_ALIGN;
  const int S = c->d.sink_frames, L = c->d.window_frames;
  const int room = (S - c->sink_held) + (L - c->win_held);
  if (n_frames > room) return ASTRO_ERR_CAPACITY;
  if (n_frames == 0) return ASTRO_OK;
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  int* slots = new (std::nothrow) int[n_frames];
  if (!slots) return ASTRO_ERR_CUDA;
  int sink = c->sink_held, held = c->win_held;
  for (int j = 0; j < n_frames; ++j) {
    if (sink < S) slots[j] = sink++;
    else { slots[j] = S + (c->win_head + held) % L; ++held; }
  }
  s = launch_ring_copy<true>(c, const_cast<void*>(k), const_cast<void*>(v), slots, n_frames,
                             static_cast<cudaStream_t>(stream));
  delete[] slots;
  if (s != ASTRO_OK) return s;
  c->sink_held = sink;
  c->win_held = held;
  c->frames_seen += n_frames;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_evict(astro_kvcache_t* c, int n_frames, void* /*stream*/) {
  if (!c) return ASTRO_ERR_NULL;
  if (n_frames < 0) return ASTRO_ERR_SHAPE;
  if (n_frames > c->win_held) return ASTRO_ERR_UNDERFLOW;
  c->win_head = (c->win_head + n_frames) % c->d.window_frames;
  c->win_held -= n_frames;
  if (c->win_held == 0) c->win_head = 0;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_query(const astro_kvcache_t* c, int* sink_held, int* window_held, int64_t* frames_seen) {
  if (!c) return ASTRO_ERR_NULL;
  if (sink_held) *sink_held = c->sink_held;
  if (window_held) *window_held = c->win_held;
  if (frames_seen) *frames_seen = c->frames_seen;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_get_state(const astro_kvcache_t* c, astro_kvcache_state_t* state) {
  if (!c || !state) return ASTRO_ERR_NULL;
  state->sink_held = c->sink_held;
  state->window_head = c->win_head;
  state->window_held = c->win_held;
  state->frames_seen = c->frames_seen;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_set_state(astro_kvcache_t* c, const astro_kvcache_state_t* state) {
  if (!c || !state) return ASTRO_ERR_NULL;
  const int S = c->d.sink_frames, L = c->d.window_frames;
  if (state->sink_held < 0 || state->sink_held > S || state->window_held < 0 || state->window_held > L ||
      state->window_head < 0 || state->window_head >= L || state->frames_seen < state->sink_held + state->window_held)
    return ASTRO_ERR_SHAPE;
  if (state->window_held > 0 && state->sink_held != S) return ASTRO_ERR_SHAPE;  // the sink fills first
  c->sink_held = state->sink_held;
  c->win_head = state->window_held == 0 ? 0 : state->window_head;
  c->win_held = state->window_held;
  c->frames_seen = state->frames_seen;
  return ASTRO_OK;
}

astro_status_t astro_kvcache_key_segments(const astro_kvcache_t* c, int n_kc, int* n_segments, int* first_token,
                                          int* token_count, int* from_chunk) {
  if (!n_segments || !first_token || !token_count || !from_chunk) return ASTRO_ERR_NULL;
  if (n_kc < 0) return ASTRO_ERR_SHAPE;
  const bool have_ctx = c && (c->sink_held + c->win_held) > 0;
  const KeySegs s = build_segments(have_ctx ? c : nullptr, n_kc);
  *n_segments = s.n;
  for (int i = 0; i < s.n; ++i) {
    first_token[i] = s.start[i];
    token_count[i] = s.count[i];
    from_chunk[i] = s.from_chunk[i];
  }
  return ASTRO_OK;
}

astro_status_t astro_kvcache_export(const astro_kvcache_t* c, void* k_out, void* v_out, void* stream) {
  if (!c || !k_out || !v_out) return ASTRO_ERR_NULL;
  if (!aligned16(k_out) || !aligned16(v_out)) return ASTRO_ERR_ALIGN;
  const int n = c->sink_held + c->win_held;
  if (n == 0) return ASTRO_OK;
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  int* slots = new (std::nothrow) int[n];
  if (!slots) return ASTRO_ERR_CUDA;
  for (int j = 0; j < c->sink_held; ++j) slots[j] = j;
  for (int j = 0; j < c->win_held; ++j)
    slots[c->sink_held + j] = c->d.sink_frames + (c->win_head + j) % c->d.window_frames;
  s = launch_ring_copy<false>(c, k_out, v_out, slots, n, static_cast<cudaStream_t>(stream));
  delete[] slots;
  return s;
}

astro_status_t astro_chunk_attn_fwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                    const void* v_chunk, int batch, int heads, int head_dim, int n_q, int n_kc,
                                    float scale, void* o, float* lse, void* stream) {
  if (!q || !o) return ASTRO_ERR_NULL;
  if (n_kc > 0 && (!k_chunk || !v_chunk)) return ASTRO_ERR_NULL;
  const AttnArgs a{cache, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(a, scale);
  if (s != ASTRO_OK) return s;
  if (!aligned16(q) || !aligned16(o) || (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk))) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return ASTRO_ERR_ALIGN;
  s = check_arch();
  if (s != ASTRO_OK) return s;
  const bool have_ctx = cache && (cache->sink_held + cache->win_held) > 0;
  CUtensorMap tkc, tvc, tkx, tvx[2];
  std::memset(&tkc, 0, sizeof(tkc)); std::memset(&tvc, 0, sizeof(tvc));
  std::memset(&tkx, 0, sizeof(tkx)); std::memset(tvx, 0, sizeof(tvx));
  if (n_kc > 0) {
    if ((s = make_tmap_user(&tkc, k_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
    if ((s = make_tmap_user(&tvc, v_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
  }
  const KeySegs segs = build_segments(have_ctx ? cache : nullptr, n_kc);
  if (have_ctx) {
    if ((s = cache_maps(cache)) != ASTRO_OK) return s;
    tkx = cache->tm_k;
    // V of each cache key range through a map that ends where the range ends: rows past it are zero-filled by
    // TMA instead of carrying whatever an evicted or never written slot holds (0 * NaN would reach O)
    for (int i = 0, ci = 0; i < segs.n; ++i) {
      if (segs.from_chunk[i]) continue;
      const long long end = static_cast<long long>(segs.start[i]) + segs.count[i];
      if ((s = make_tmap_cache_range(&tvx[ci++], cache, cache->v, end, kTile)) != ASTRO_OK) return s;
    }
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(q);
  if (head_dim == 128 && g_fwd_mode.load(std::memory_order_relaxed) == 2)
    return launch_fwd_pair(a, cache, have_ctx, q, k_chunk, v_chunk, segs, scale, o, lse, st);
  return head_dim == 128 ? launch_fwd<128>(a, qp, tkc, tvc, tkx, tvx, segs, scale, o, lse, st)
                         : launch_fwd<64>(a, qp, tkc, tvc, tkx, tvx, segs, scale, o, lse, st);
}

size_t astro_chunk_attn_bwd_workspace_bytes(int batch, int heads, int n_q, int head_dim) {
  if (batch < 1 || heads < 1 || n_q < 1 || (head_dim != 64 && head_dim != 128)) return 0;
  const size_t b = static_cast<size_t>(batch) * heads * n_q * sizeof(float);
  return (b + 255) & ~static_cast<size_t>(255);
}

astro_status_t astro_chunk_attn_bwd_delta(const void* o, const void* d_o, int batch, int heads, int head_dim, int n_q,
                                          float* delta, void* stream) {
  if (!o || !d_o || !delta) return ASTRO_ERR_NULL;
  if (batch < 1 || heads < 1 || n_q < 1 || (head_dim != 64 && head_dim != 128)) return ASTRO_ERR_SHAPE;
  if (!aligned16(o) || !aligned16(d_o) || !aligned16(delta)) return ASTRO_ERR_ALIGN;
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_bwd_delta<128>(o, d_o, batch, heads, n_q, delta, st)
                         : launch_bwd_delta<64>(o, d_o, batch, heads, n_q, delta, st);
}

astro_status_t astro_chunk_attn_bwd_dq(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                       const void* v_chunk, const float* lse, const float* delta, const void* d_o,
                                       int batch, int heads, int head_dim, int n_q, int n_kc, float scale, void* dq,
                                       void* stream) {
  if (!q || !lse || !delta || !d_o || !dq) return ASTRO_ERR_NULL;
  if (n_kc > 0 && (!k_chunk || !v_chunk)) return ASTRO_ERR_NULL;
  const AttnArgs a{cache, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(a, scale);
  if (s != ASTRO_OK) return s;
  if (!aligned16(q) || !aligned16(d_o) || !aligned16(dq) || (reinterpret_cast<uintptr_t>(lse) & 3u) ||
      (reinterpret_cast<uintptr_t>(delta) & 3u) || (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk))))
    return ASTRO_ERR_ALIGN;
  s = check_arch();
  if (s != ASTRO_OK) return s;
  const bool have_ctx = cache && (cache->sink_held + cache->win_held) > 0;
  CUtensorMap tdo, tkc, tvc, tkx[2], tvx;
  std::memset(&tkc, 0, sizeof(tkc)); std::memset(&tvc, 0, sizeof(tvc));
  std::memset(tkx, 0, sizeof(tkx)); std::memset(&tvx, 0, sizeof(tvx));
  if ((s = make_tmap_user(&tdo, d_o, head_dim, n_q, heads, batch)) != ASTRO_OK) return s;
  if (n_kc > 0) {
    if ((s = make_tmap_user(&tkc, k_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
    if ((s = make_tmap_user(&tvc, v_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
  }
  const KeySegs segs = build_segments(have_ctx ? cache : nullptr, n_kc);
  if (have_ctx) {
    if ((s = cache_maps(cache)) != ASTRO_OK) return s;
    tvx = cache->tm_v;
    // K of each cache key range through a map that ends where the range ends (rows past it are zeros: dS is 0
    // there, but 0 * NaN from a stale slot would reach dQ)
    for (int i = 0, ci = 0; i < segs.n; ++i) {
      if (segs.from_chunk[i]) continue;
      const long long end = static_cast<long long>(segs.start[i]) + segs.count[i];
      if ((s = make_tmap_cache_range(&tkx[ci++], cache, cache->k, end, kTile)) != ASTRO_OK) return s;
    }
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(q);
  return head_dim == 128 ? launch_bwd_dq<128>(a, qp, tdo, tkc, tvc, tkx, tvx, segs, scale, lse, delta, dq, st)
                         : launch_bwd_dq<64>(a, qp, tdo, tkc, tvc, tkx, tvx, segs, scale, lse, delta, dq, st);
}

astro_status_t astro_chunk_attn_bwd_dkv(const void* q, const void* k_chunk, const void* v_chunk, const float* lse,
                                        const float* delta, const void* d_o, int batch, int heads, int head_dim,
                                        int n_q, int n_kc, float scale, void* dk_chunk, void* dv_chunk, void* stream) {
  if (!q || !k_chunk || !v_chunk || !lse || !delta || !d_o || !dk_chunk || !dv_chunk) return ASTRO_ERR_NULL;
  const AttnArgs a{nullptr, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(a, scale);
  if (s != ASTRO_OK) return s;
  if (!aligned16(q) || !aligned16(d_o) || !aligned16(k_chunk) || !aligned16(v_chunk) || !aligned16(dk_chunk) ||
      !aligned16(dv_chunk) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(delta) & 3u))
    return ASTRO_ERR_ALIGN;
  s = check_arch();
  if (s != ASTRO_OK) return s;
  CUtensorMap tq, tdo, tkc, tvc;
  if ((s = make_tmap_user(&tq, q, head_dim, n_q, heads, batch)) != ASTRO_OK) return s;
  if ((s = make_tmap_user(&tdo, d_o, head_dim, n_q, heads, batch)) != ASTRO_OK) return s;
  if ((s = make_tmap_user(&tkc, k_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
  if ((s = make_tmap_user(&tvc, v_chunk, head_dim, n_kc, heads, batch)) != ASTRO_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_bwd_dkv<128>(a, tq, tdo, tkc, tvc, scale, lse, delta, dk_chunk, dv_chunk, st)
                         : launch_bwd_dkv<64>(a, tq, tdo, tkc, tvc, scale, lse, delta, dk_chunk, dv_chunk, st);
}

astro_status_t astro_chunk_attn_bwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                    const void* v_chunk, const void* o, const float* lse, const void* d_o, int batch,
                                    int heads, int head_dim, int n_q, int n_kc, float scale, void* dq, void* dk_chunk,
                                    void* dv_chunk, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !o || !lse || !d_o || !dq || !workspace) return ASTRO_ERR_NULL;
  if (n_kc > 0 && (!k_chunk || !v_chunk || !dk_chunk || !dv_chunk)) return ASTRO_ERR_NULL;
  const AttnArgs a{cache, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(a, scale);
  if (s != ASTRO_OK) return s;
  if (workspace_bytes < astro_chunk_attn_bwd_workspace_bytes(batch, heads, n_q, head_dim)) return ASTRO_ERR_CAPACITY;
  if (!aligned16(q) || !aligned16(o) || !aligned16(d_o) || !aligned16(dq) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u) ||
      (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk) || !aligned16(dk_chunk) || !aligned16(dv_chunk))))
    return ASTRO_ERR_ALIGN;
  float* delta = static_cast<float*>(workspace);
  s = astro_chunk_attn_bwd_delta(o, d_o, batch, heads, head_dim, n_q, delta, stream);
  if (s != ASTRO_OK) return s;
  s = astro_chunk_attn_bwd_dq(cache, q, k_chunk, v_chunk, lse, delta, d_o, batch, heads, head_dim, n_q, n_kc, scale,
                              dq, stream);
  if (s != ASTRO_OK || n_kc == 0) return s;
  return astro_chunk_attn_bwd_dkv(q, k_chunk, v_chunk, lse, delta, d_o, batch, heads, head_dim, n_q, n_kc, scale,
                                  dk_chunk, dv_chunk, stream);
}

astro_status_t astro_kvcache_fork(astro_kvcache_t* dst, const astro_kvcache_t* src, const int32_t* parents,
                                  const int* frames, int n_frames, void* stream) {
  if (!dst || !src || (!frames && n_frames > 0)) return ASTRO_ERR_NULL;
  const auto &a = src->d, &d = dst->d;
  const int held = src->sink_held + src->win_held;
  if (!frames && n_frames == -1) n_frames = held;
  if (n_frames < 0 || dst == src || a.heads != d.heads || a.head_dim != d.head_dim ||
      a.tokens_per_frame != d.tokens_per_frame)
    return ASTRO_ERR_SHAPE;
  if (!parents && a.cache_batch != 1 && a.cache_batch != d.cache_batch) return ASTRO_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(parents) & 3u) return ASTRO_ERR_ALIGN;
  const size_t src_bytes = astro_kvcache_storage_bytes(&a), dst_bytes = astro_kvcache_storage_bytes(&d);
  const uintptr_t from[2] = {reinterpret_cast<uintptr_t>(src->k), reinterpret_cast<uintptr_t>(src->v)};
  const uintptr_t to[2] = {reinterpret_cast<uintptr_t>(dst->k), reinterpret_cast<uintptr_t>(dst->v)};
  for (uintptr_t f : from)
    for (uintptr_t t : to)
      if (f < t + dst_bytes && t < f + src_bytes) return ASTRO_ERR_SHAPE;
  if (n_frames > static_cast<long long>(d.sink_frames) + d.window_frames) return ASTRO_ERR_CAPACITY;
  for (int j = 0; frames && j < n_frames; ++j)
    if (frames[j] < 0 || frames[j] >= held) return ASTRO_ERR_SHAPE;
  const long long frame_vecs = static_cast<long long>(d.tokens_per_frame) * d.head_dim / 8;
  const long long pieces = (frame_vecs + kForkThreads * kForkVecsPerThread - 1) / (kForkThreads * kForkVecsPerThread);
  const long long per_frame = 2ll * d.cache_batch * d.heads * pieces;
  if (frame_vecs > 0x3fffffffLL || per_frame > 0x7fffffffLL) return ASTRO_ERR_SHAPE;
  if (n_frames > 0) {
    astro_status_t s = check_arch();
    if (s != ASTRO_OK) return s;
    // as many frames per launch as the map and the grid take
    const long long most = 0x7fffffffLL / per_frame;
    const int step = most < kMaxFramesPerCopy ? static_cast<int>(most) : kMaxFramesPerCopy;
    for (int f0 = 0; f0 < n_frames; f0 += step) {
      ForkMap map;
      map.n = n_frames - f0 < step ? n_frames - f0 : step;
      for (int j = 0; j < map.n; ++j) {
        const int f = frames ? frames[f0 + j] : f0 + j;
        map.from[j] = f < src->sink_held ? f : a.sink_frames + (src->win_head + f - src->sink_held) % a.window_frames;
        map.to[j] = f0 + j;   // an emptied cache fills its sink and then the window from ring index 0
      }
      cache_fork_kernel<<<static_cast<unsigned>(map.n * per_frame), kForkThreads, 0, static_cast<cudaStream_t>(stream)>>>(
          static_cast<const uint4*>(src->k), static_cast<const uint4*>(src->v), static_cast<uint4*>(dst->k),
          static_cast<uint4*>(dst->v), parents, map, a.cache_batch, d.cache_batch, d.heads, static_cast<int>(frame_vecs),
          static_cast<int>(pieces), a.sink_frames + a.window_frames, d.sink_frames + d.window_frames);
    }
    if ((s = launch_status()) != ASTRO_OK) return s;
  }
  dst->sink_held = n_frames < d.sink_frames ? n_frames : d.sink_frames;
  dst->win_head = 0;
  dst->win_held = n_frames - dst->sink_held;
  dst->frames_seen = src->frames_seen > n_frames ? src->frames_seen : n_frames;
  return ASTRO_OK;
}

// ---- rotary positions -------------------------------------------------------------------------------
astro_status_t astro_rope_create(const astro_rope_desc_t* d, astro_rope_t** out) {
  if (!d || !out) return ASTRO_ERR_NULL;
  if (d->head_dim < 8 || d->head_dim > 2 * kRopeMaxPairs || d->head_dim % 8 || d->rot_dim < 2 || d->rot_dim % 2 ||
      d->rot_dim > d->head_dim || d->axes < 1 || d->axes > 4)
    return ASTRO_ERR_SHAPE;
  if (d->layout != ASTRO_ROPE_INTERLEAVED && d->layout != ASTRO_ROPE_HALVES) return ASTRO_ERR_SHAPE;
  if (d->scaling < ASTRO_ROPE_SCALE_NONE || d->scaling > ASTRO_ROPE_SCALE_RAMP) return ASTRO_ERR_SHAPE;
  if (!(d->base > 0.0) || !std::isfinite(d->base) || !(d->magnitude >= 0.0) || !std::isfinite(d->magnitude))
    return ASTRO_ERR_SHAPE;
  if (d->scaling != ASTRO_ROPE_SCALE_NONE && (!(d->factor >= 1.0) || !std::isfinite(d->factor))) return ASTRO_ERR_SHAPE;
  if (d->scaling == ASTRO_ROPE_SCALE_RAMP &&
      (!(d->original_length > 0.0) || !std::isfinite(d->original_length) || !(d->ramp_low < d->ramp_high) ||
       !std::isfinite(d->ramp_low) || !std::isfinite(d->ramp_high)))
    return ASTRO_ERR_SHAPE;
  long long sum = 0;
  for (int a = 0; a < d->axes; ++a) {
    if (d->axis_pairs[a] < 1) return ASTRO_ERR_SHAPE;
    sum += d->axis_pairs[a];
  }
  if (sum != d->rot_dim / 2) return ASTRO_ERR_SHAPE;
  astro_rope* r = new (std::nothrow) astro_rope();
  if (!r) return ASTRO_ERR_CUDA;
  r->d = *d;
  const double two_pi = 6.283185307179586476925286766559;
  int p = 0;
  bool numbers = true;   // an infinite or vanished frequency turns positions, 0 among them, into NaN or into none
  for (int a = 0; a < d->axes; ++a) {
    const int n = d->axis_pairs[a];
    const bool scaled = d->scaling != ASTRO_ROPE_SCALE_NONE && ((d->scaled_axes >> a) & 1);
    double base = d->base;
    if (scaled && d->scaling == ASTRO_ROPE_SCALE_BASE && n > 1) base *= std::pow(d->factor, static_cast<double>(n) / (n - 1));
    for (int i = 0; i < n; ++i, ++p) {
      double f = std::pow(base, -static_cast<double>(i) / n);
      if (scaled && d->scaling == ASTRO_ROPE_SCALE_LINEAR) f /= d->factor;
      if (scaled && d->scaling == ASTRO_ROPE_SCALE_RAMP) {
        double g = (d->original_length * f / two_pi - d->ramp_low) / (d->ramp_high - d->ramp_low);
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        f *= g + (1.0 - g) / d->factor;
      }
      numbers = numbers && f > 0.0 && std::isfinite(f) && std::isfinite(base);
      r->frequency[p] = f;
      r->table.turns[p] = f / two_pi;
      r->table.axis[p] = static_cast<uint8_t>(a);
    }
  }
  r->magnitude = d->magnitude > 0.0 ? d->magnitude
                                    : d->scaling == ASTRO_ROPE_SCALE_RAMP ? 0.1 * std::log(d->factor) + 1.0 : 1.0;
  r->table.size = static_cast<float>(r->magnitude);
  if (!numbers || !(r->table.size > 0.f) || !std::isfinite(r->table.size)) {
    delete r;
    return ASTRO_ERR_SHAPE;
  }
  r->table.pairs = p;
  r->table.axes = d->axes;
  *out = r;
  return ASTRO_OK;
}

astro_status_t astro_rope_destroy(astro_rope_t* rope) {
  if (!rope) return ASTRO_ERR_NULL;
  delete rope;
  return ASTRO_OK;
}

astro_status_t astro_rope_frequencies(const astro_rope_t* rope, double* frequencies, double* magnitude) {
  if (!rope || !frequencies) return ASTRO_ERR_NULL;
  std::memcpy(frequencies, rope->frequency, sizeof(double) * rope->table.pairs);
  if (magnitude) *magnitude = rope->magnitude;
  return ASTRO_OK;
}

static astro_status_t check_rope(const astro_rope_t* rope, int inverse, const void* q, const void* k, const int32_t* positions,
                                 int positions_batch, int batch, int n_tokens, int heads_q, int heads_k, int dtype,
                                 const astro_strides_t* in_strides, void* q_out, void* k_out, const astro_strides_t* out_strides,
                                 RopeTensors* x) {
  if (!rope || (k != nullptr) != (k_out != nullptr)) return ASTRO_ERR_NULL;
  if (batch < 1 || n_tokens < 0 || heads_q < 1 || (k && heads_k < 1) || (positions_batch != 1 && positions_batch != batch))
    return ASTRO_ERR_SHAPE;
  if (dtype != ASTRO_BF16 && dtype != ASTRO_F16 && dtype != ASTRO_F32) return ASTRO_ERR_SHAPE;
  if (inverse != 0 && inverse != 1) return ASTRO_ERR_SHAPE;
  if (static_cast<long long>(batch) * n_tokens > 0x7fffffffLL || heads_q > 65535 || (k && heads_k > 65535))
    return ASTRO_ERR_SHAPE;
  if (n_tokens == 0) return ASTRO_OK;
  if (!q || !q_out || !positions) return ASTRO_ERR_NULL;
  const int size = dtype == ASTRO_F32 ? 4 : 2, per16 = 16 / size, D = rope->d.head_dim;
  if (!aligned16(q) || !aligned16(q_out) || (k && (!aligned16(k) || !aligned16(k_out))) ||
      (reinterpret_cast<uintptr_t>(positions) & 3u))
    return ASTRO_ERR_ALIGN;
  const int heads = k && heads_k > heads_q ? heads_k : heads_q;
  // contiguous tensors of different head counts have different strides: those need two calls
  if (k && heads_k != heads_q && (!in_strides || !out_strides)) return ASTRO_ERR_SHAPE;
  const astro_strides_t dense = {static_cast<int64_t>(n_tokens) * heads_q * D, static_cast<int64_t>(heads_q) * D, D};
  const astro_strides_t in = in_strides ? *in_strides : dense, to = out_strides ? *out_strides : dense;
  const long long sizes[3] = {batch, n_tokens, heads}, is[3] = {in.batch, in.token, in.head}, os[3] = {to.batch, to.token, to.head};
  const long long limit = 1ll << 40;   // elements from the first row to the last along an axis: beyond any memory, sums inside 64 bits
  for (int i = 0; i < 3; ++i) {
    if (sizes[i] <= 1) continue;
    const long long most = limit / (sizes[i] - 1);
    if (is[i] < 0 || os[i] < 0 || is[i] > most || os[i] > most) return ASTRO_ERR_SHAPE;
    if (is[i] % per16 || os[i] % per16) return ASTRO_ERR_ALIGN;
  }
  if (overlaps_itself(sizes, os, D)) return ASTRO_ERR_SHAPE;
  if (q_out == k_out || (k && (q_out == k || k_out == q))) return ASTRO_ERR_SHAPE;
  if (q_out == q || (k && k_out == k))
    for (int i = 0; i < 3; ++i)
      if (sizes[i] > 1 && is[i] != os[i]) return ASTRO_ERR_SHAPE;
  x->q = q; x->k = k; x->q_out = q_out; x->k_out = k_out;
  x->heads_q = heads_q;
  x->heads_k = k ? heads_k : 0;
  x->in_b = in.batch; x->in_t = in.token; x->in_h = in.head;
  x->out_b = to.batch; x->out_t = to.token; x->out_h = to.head;
  return ASTRO_OK;
}

astro_status_t astro_rope_apply_check(const astro_rope_t* rope, int inverse, const void* q, const void* k,
                                      const int32_t* positions, int positions_batch, int batch, int n_tokens, int heads_q,
                                      int heads_k, int dtype, const astro_strides_t* in_strides, void* q_out, void* k_out,
                                      const astro_strides_t* out_strides) {
  RopeTensors x;
  return check_rope(rope, inverse, q, k, positions, positions_batch, batch, n_tokens, heads_q, heads_k, dtype, in_strides, q_out,
                    k_out, out_strides, &x);
}

astro_status_t astro_rope_apply(const astro_rope_t* rope, int inverse, const void* q, const void* k,
                                const int32_t* positions, int positions_batch, int batch, int n_tokens, int heads_q,
                                int heads_k, int dtype, const astro_strides_t* in_strides, void* q_out, void* k_out,
                                const astro_strides_t* out_strides, void* stream) {
  RopeTensors x;
  astro_status_t s = check_rope(rope, inverse, q, k, positions, positions_batch, batch, n_tokens, heads_q, heads_k, dtype,
                                in_strides, q_out, k_out, out_strides, &x);
  if (s != ASTRO_OK || n_tokens == 0) return s;
  if ((s = check_arch()) != ASTRO_OK) return s;
  const int total = batch * n_tokens, per_sample = positions_batch > 1 || batch == 1 ? 1 : 0;
  const float sign = inverse ? -1.f : 1.f;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == ASTRO_BF16) return launch_rope_typed<__nv_bfloat16>(rope, x, positions, per_sample, n_tokens, total, sign, st);
  if (dtype == ASTRO_F16) return launch_rope_typed<__half>(rope, x, positions, per_sample, n_tokens, total, sign, st);
  return launch_rope_typed<float>(rope, x, positions, per_sample, n_tokens, total, sign, st);
}

// ---- key blocks ---------------------------------------------------------------------------------------
astro_status_t astro_block_count(const astro_kvcache_t* cache, int n_kc, int block_tokens, int* ctx_blocks,
                                 int* chunk_blocks) {
  KeyBlocks kb;
  if (!block_tokens_ok(block_tokens) || n_kc < 0 || !build_key_blocks(cache, n_kc, block_tokens, &kb)) return ASTRO_ERR_SHAPE;
  if (ctx_blocks) *ctx_blocks = kb.ctx;
  if (chunk_blocks) *chunk_blocks = kb.total - kb.ctx;
  return ASTRO_OK;
}

astro_status_t astro_block_pool(const astro_kvcache_t* c, int first_frame, int n_frames, int block_tokens, float* pooled,
                                void* stream) {
  if (!c || !pooled) return ASTRO_ERR_NULL;
  KeyBlocks kb;
  if (!block_tokens_ok(block_tokens) || !build_key_blocks(c, 0, block_tokens, &kb)) return ASTRO_ERR_SHAPE;
  const int held = c->sink_held + c->win_held;
  if (first_frame < 0 || n_frames < 0 || first_frame > held || n_frames > held - first_frame) return ASTRO_ERR_SHAPE;
  if (!aligned16(pooled)) return ASTRO_ERR_ALIGN;
  const auto& d = c->d;
  if (d.heads > 65535 || d.cache_batch > 65535) return ASTRO_ERR_SHAPE;
  if (n_frames == 0) return ASTRO_OK;
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  const long long slots = d.sink_frames + d.window_frames;
  PoolSource src;
  src.base = static_cast<const __nv_bfloat16*>(c->k);
  src.st = d.head_dim;
  src.sh = slots * d.tokens_per_frame * d.head_dim;
  src.sb = src.sh * d.heads;
  src.out = pooled;
  src.out_h = slots * kb.per_frame;
  src.out_b = src.out_h * d.heads;
  src.tokens = d.tokens_per_frame;
  src.block = block_tokens;
  src.blocks = n_frames * kb.per_frame;
  set_inverses(&src);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return d.head_dim == 128 ? launch_pool<128>(src, d.heads, d.cache_batch, kb, first_frame, st)
                           : launch_pool<64>(src, d.heads, d.cache_batch, kb, first_frame, st);
}

size_t astro_block_select_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_kc, int block_tokens) {
  if (batch < 1 || heads < 1 || n_q < 1 || n_kc < 0 || (head_dim != 64 && head_dim != 128) || !block_tokens_ok(block_tokens))
    return 0;
  const size_t blocks = static_cast<size_t>((n_q - 1) / ASTRO_QUERY_BLOCK + 1) + (static_cast<size_t>(n_kc) + block_tokens - 1) / block_tokens;
  return blocks * batch * heads * head_dim * sizeof(float);
}

astro_status_t astro_block_select(const astro_kvcache_t* cache, const float* pooled, const void* q, const void* k_chunk,
                                  int batch, int heads, int head_dim, int n_q, int n_kc, int block_tokens, int n_select,
                                  int keep, int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !blocks || !workspace || (n_kc > 0 && !k_chunk)) return ASTRO_ERR_NULL;
  const AttnArgs args{cache, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(args, 1.f);
  if (s != ASTRO_OK) return s;
  KeyBlocks kb;
  if (!block_tokens_ok(block_tokens) || n_select < 1 || n_select > ASTRO_MAX_SELECT || (keep & ~(ASTRO_KEEP_SINK | ASTRO_KEEP_CHUNK)) ||
      !build_key_blocks(cache, n_kc, block_tokens, &kb) || kb.total > ASTRO_SELECT_MAX_BLOCKS)
    return ASTRO_ERR_SHAPE;
  if (kb.ctx > 0 && !pooled) return ASTRO_ERR_NULL;
  if (!aligned16(q) || (n_kc > 0 && !aligned16(k_chunk)) || !aligned16(pooled) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(blocks) & 3u))
    return ASTRO_ERR_ALIGN;
  if (workspace_bytes < astro_block_select_workspace_bytes(batch, heads, head_dim, n_q, n_kc, block_tokens))
    return ASTRO_ERR_CAPACITY;
  if ((s = check_arch()) != ASTRO_OK) return s;
  const long long row = static_cast<long long>(heads) * head_dim;
  PoolSource qs, ks;
  qs.base = static_cast<const __nv_bfloat16*>(q);
  qs.st = row; qs.sh = head_dim; qs.sb = row * n_q;
  qs.tokens = n_q;
  qs.block = ASTRO_QUERY_BLOCK;
  qs.blocks = (n_q - 1) / ASTRO_QUERY_BLOCK + 1;
  set_inverses(&qs);
  qs.out = static_cast<float*>(workspace);
  qs.out_h = qs.blocks;
  qs.out_b = qs.out_h * heads;
  ks = qs;
  ks.base = static_cast<const __nv_bfloat16*>(k_chunk);
  ks.sb = row * n_kc;
  ks.tokens = n_kc;
  ks.block = block_tokens;
  ks.blocks = kb.total - kb.ctx;
  set_inverses(&ks);
  ks.out = qs.out + qs.out_b * batch * head_dim;
  ks.out_h = ks.blocks;
  ks.out_b = ks.out_h * heads;
  SelectArgs a;
  a.pooled = pooled;
  a.q_mean = qs.out;
  a.kc_mean = ks.out;
  a.blocks = blocks;
  a.heads = heads;
  a.q_blocks = qs.blocks;
  a.n_select = n_select;
  a.cache_shared = cache && cache->d.cache_batch == 1 && batch > 1;
  a.keep_sink = keep & ASTRO_KEEP_SINK ? 1 : 0;
  a.keep_chunk = keep & ASTRO_KEEP_CHUNK ? 1 : 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_select<128>(qs, ks, a, kb, batch, st) : launch_select<64>(qs, ks, a, kb, batch, st);
}

size_t astro_sparse_attn_fwd_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_select, int block_tokens) {
  if (batch < 1 || heads < 1 || n_q < 1 || n_select < 1 || (head_dim != 64 && head_dim != 128) || !block_tokens_ok(block_tokens))
    return 0;
  const SparseSplit sp = sparse_split(batch, heads, n_q, n_select, block_tokens);
  return sp.splits == 1 ? 0 : static_cast<size_t>(sp.splits) * batch * heads * n_q * (head_dim + 1) * sizeof(float);
}

astro_status_t astro_sparse_attn_fwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk,
                                     const int32_t* blocks, int n_select, int block_tokens, int batch, int heads,
                                     int head_dim, int n_q, int n_kc, float scale, void* o, float* lse, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  if (!q || !o || !blocks || (n_kc > 0 && (!k_chunk || !v_chunk))) return ASTRO_ERR_NULL;
  const SparseCall c{{cache, batch, heads, head_dim, n_q, n_kc}, q, k_chunk, v_chunk, blocks, n_select, block_tokens};
  SparseGeom g;
  astro_status_t s = check_sparse(c, scale, &g);
  if (s != ASTRO_OK) return s;
  const size_t need = astro_sparse_attn_fwd_workspace_bytes(batch, heads, head_dim, n_q, n_select, block_tokens);
  if (need > 0 && !workspace) return ASTRO_ERR_NULL;
  if (!aligned16(q) || !aligned16(o) || (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk))) ||
      (need > 0 && !aligned16(workspace)) || (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(blocks) & 3u))
    return ASTRO_ERR_ALIGN;
  if (workspace_bytes < need) return ASTRO_ERR_CAPACITY;
  if ((s = check_arch()) != ASTRO_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_sparse_fwd<128>(c, g, scale, o, lse, workspace, st)
                         : launch_sparse_fwd<64>(c, g, scale, o, lse, workspace, st);
}

size_t astro_sparse_attn_bwd_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_kc, int n_select,
                                             int block_tokens) {
  if (batch < 1 || heads < 1 || n_q < 1 || n_kc < 0 || n_select < 1 || (head_dim != 64 && head_dim != 128) ||
      !block_tokens_ok(block_tokens))
    return 0;
  const SparseBwdScratch s = sparse_bwd_scratch(batch, heads, n_q, n_kc, block_tokens);
  return s.delta + s.counts;
}

astro_status_t astro_sparse_attn_bwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk,
                                     const int32_t* blocks, int n_select, int block_tokens, const void* o, const float* lse,
                                     const void* d_o, int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                     void* dq, void* dk_chunk, void* dv_chunk, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  if (!q || !blocks || !o || !lse || !d_o || !dq || !workspace) return ASTRO_ERR_NULL;
  if (n_kc > 0 && (!k_chunk || !v_chunk || !dk_chunk || !dv_chunk)) return ASTRO_ERR_NULL;
  const SparseCall c{{cache, batch, heads, head_dim, n_q, n_kc}, q, k_chunk, v_chunk, blocks, n_select, block_tokens};
  SparseGeom g;
  astro_status_t s = check_sparse(c, scale, &g);
  if (s != ASTRO_OK) return s;
  const long long q_tiles = (n_q - 1) / kTile + 1;
  if (q_tiles * n_select > 0x3fffffffLL) return ASTRO_ERR_SHAPE;   // the tiles of a block are counted in 32 bits
  if (!aligned16(q) || !aligned16(o) || !aligned16(d_o) || !aligned16(dq) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u) || (reinterpret_cast<uintptr_t>(blocks) & 3u) ||
      (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk) || !aligned16(dk_chunk) || !aligned16(dv_chunk))))
    return ASTRO_ERR_ALIGN;
  if (workspace_bytes < astro_sparse_attn_bwd_workspace_bytes(batch, heads, head_dim, n_q, n_kc, n_select, block_tokens))
    return ASTRO_ERR_CAPACITY;
  if ((s = check_arch()) != ASTRO_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return head_dim == 128 ? launch_sparse_bwd<128>(c, g, scale, o, lse, d_o, dq, dk_chunk, dv_chunk, workspace, st)
                         : launch_sparse_bwd<64>(c, g, scale, o, lse, d_o, dq, dk_chunk, dv_chunk, workspace, st);
}

astro_status_t astro_nft_loss(const void* v_theta, const void* v_old, const void* v_ref, const void* v_target,
                              const float* r_tilde, const float* w_policy, const float* w_kl, int batch,
                              long long elems, float beta, float* policy_out, float* kl_out, void* grad,
                              void* stream) {
  if (!v_theta || !v_old || !v_target || !r_tilde || !policy_out) return ASTRO_ERR_NULL;
  if ((v_ref == nullptr) != (kl_out == nullptr)) return ASTRO_ERR_NULL;
  if (batch < 1 || batch > 65535 || elems < 8 || (elems & 7)) return ASTRO_ERR_SHAPE;
  if (!aligned16(v_theta) || !aligned16(v_old) || !aligned16(v_target) || (v_ref && !aligned16(v_ref)) ||
      (grad && !aligned16(grad)))
    return ASTRO_ERR_ALIGN;
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cudaMemsetAsync(policy_out, 0, sizeof(float) * batch, st) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (kl_out && cudaMemsetAsync(kl_out, 0, sizeof(float) * batch, st) != cudaSuccess) return ASTRO_ERR_CUDA;
  const long long vecs = elems / 8;
  const long long per_block = static_cast<long long>(kNftThreads) * kNftVecsPerThread;
  long long blocks = (vecs + per_block - 1) / per_block;
  if (blocks > 4096) blocks = 4096;
  dim3 grid(static_cast<unsigned>(blocks), batch);
  nft_loss_kernel<<<grid, kNftThreads, 0, st>>>(
      static_cast<const uint4*>(v_theta), static_cast<const uint4*>(v_old), static_cast<const uint4*>(v_ref),
      static_cast<const uint4*>(v_target), r_tilde, w_policy, w_kl, vecs, beta, policy_out, kl_out,
      static_cast<uint4*>(grad));
  return launch_status();
}

// ---- backward without caller scratch ---------------------------------------------------------------
// delta lives in this fixed device array.  In host code `g_bwd_static_delta` is only a stand-in for the
// symbol, not a device address: the address each GPU gives it is looked up once per device below.
static __device__ __align__(256) float g_bwd_static_delta[ASTRO_BWD_STATIC_MAX_ROWS];

static astro_status_t bwd_static_scratch(float** out) {
  static std::atomic<float*> addr[kMaxDevices];   // every thread that races here stores the same address
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return ASTRO_ERR_CUDA;
  float* p = addr[dev].load(std::memory_order_acquire);
  if (!p) {
    if (cudaGetSymbolAddress(reinterpret_cast<void**>(&p), g_bwd_static_delta) != cudaSuccess || !p)
      return ASTRO_ERR_CUDA;
    addr[dev].store(p, std::memory_order_release);
  }
  *out = p;
  return ASTRO_OK;
}

astro_status_t astro_chunk_attn_bwd_static(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                           const void* v_chunk, const void* o, const float* lse, const void* d_o,
                                           int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                           void* dq, void* dk_chunk, void* dv_chunk, void* stream) {
  if (!q || !o || !lse || !d_o || !dq) return ASTRO_ERR_NULL;
  if (n_kc > 0 && (!k_chunk || !v_chunk || !dk_chunk || !dv_chunk)) return ASTRO_ERR_NULL;
  const AttnArgs a{cache, batch, heads, head_dim, n_q, n_kc};
  astro_status_t s = check_attn_args(a, scale);
  if (s != ASTRO_OK) return s;
  if (!aligned16(q) || !aligned16(o) || !aligned16(d_o) || !aligned16(dq) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u) ||
      (n_kc > 0 && (!aligned16(k_chunk) || !aligned16(v_chunk) || !aligned16(dk_chunk) || !aligned16(dv_chunk))))
    return ASTRO_ERR_ALIGN;
  if (static_cast<long long>(batch) * heads * n_q > ASTRO_BWD_STATIC_MAX_ROWS) return ASTRO_ERR_CAPACITY;
  s = check_arch();
  if (s != ASTRO_OK) return s;
  float* delta = nullptr;
  if ((s = bwd_static_scratch(&delta)) != ASTRO_OK) return s;
  s = astro_chunk_attn_bwd_delta(o, d_o, batch, heads, head_dim, n_q, delta, stream);
  if (s != ASTRO_OK) return s;
  s = astro_chunk_attn_bwd_dq(cache, q, k_chunk, v_chunk, lse, delta, d_o, batch, heads, head_dim, n_q, n_kc, scale,
                              dq, stream);
  if (s != ASTRO_OK || n_kc == 0) return s;
  return astro_chunk_attn_bwd_dkv(q, k_chunk, v_chunk, lse, delta, d_o, batch, heads, head_dim, n_q, n_kc, scale,
                                  dk_chunk, dv_chunk, stream);
}

astro_status_t astro_debug_forward_mode(int mode) {
  if (mode < 0 || mode > 2) return ASTRO_ERR_SHAPE;
  g_fwd_mode.store(mode, std::memory_order_relaxed);
  return ASTRO_OK;
}

astro_status_t astro_debug_pair_flag(int* flag) {
  if (!flag) return ASTRO_ERR_NULL;
  if (cudaDeviceSynchronize() != cudaSuccess) return ASTRO_ERR_CUDA;
  if (cudaMemcpyFromSymbol(flag, g_pair_needs_safe, sizeof(int)) != cudaSuccess) return ASTRO_ERR_CUDA;
  const int zero = 0;
  if (cudaMemcpyToSymbol(g_pair_needs_safe, &zero, sizeof(zero)) != cudaSuccess) return ASTRO_ERR_CUDA;
  return ASTRO_OK;
}

astro_status_t astro_selftest_wait_timeout(void* stream) {
  astro_status_t s = check_arch();
  if (s != ASTRO_OK) return s;
  wait_timeout_selftest_kernel<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(2000000LL);  // about 1 ms
  return launch_status();
}

astro_status_t astro_last_device_status(uint32_t* detail) {
  if (cudaDeviceSynchronize() != cudaSuccess) return ASTRO_ERR_CUDA;
  uint32_t word = 0;
  if (cudaMemcpyFromSymbol(&word, g_device_status, sizeof(word)) != cudaSuccess) return ASTRO_ERR_CUDA;
  if (detail) *detail = word;
  if (word == 0) return ASTRO_OK;
  const uint32_t zero = 0;
  if (cudaMemcpyToSymbol(g_device_status, &zero, sizeof(zero)) != cudaSuccess) return ASTRO_ERR_CUDA;
  return ASTRO_ERR_TIMEOUT;
}

const char* astro_status_string(astro_status_t s) {
  switch (s) {
    case ASTRO_OK: return "ok";
    case ASTRO_ERR_NULL: return "null pointer";
    case ASTRO_ERR_SHAPE: return "unsupported or inconsistent shape";
    case ASTRO_ERR_ALIGN: return "pointer not 16-byte aligned";
    case ASTRO_ERR_CAPACITY: return "capacity exceeded";
    case ASTRO_ERR_UNDERFLOW: return "evict exceeds window frames held";
    case ASTRO_ERR_ARCH: return "device is not compute capability 10.x";
    case ASTRO_ERR_CUDA: return "CUDA call failed";
    case ASTRO_ERR_TIMEOUT: return "a bounded device-side wait ran out";
  }
  return "unknown status";
}

}  // extern "C"
