/*
 * astro.h -- C ABI of the rolling-KV chunk-attention library (sm_100a).
 *
 * One DiT layer's self-attention in the streaming scheme: the queries of a new
 * chunk of latent frames attend to a restricted context (S permanently kept
 * "sink" frames plus a sliding window of recent frames) and to the chunk itself.
 *
 * Conventions shared by every call
 *   - Every data pointer is a DEVICE pointer to memory the caller allocated and
 *     keeps alive; the library frees none of it.  The cache handle owns only
 *     host-side metadata.  Query outputs (int*, int64_t*) are HOST pointers.
 *   - Work is enqueued on the given CUDA stream (passed as void*, a cudaStream_t)
 *     and the call returns without synchronising.  Metadata changes take effect in
 *     call order.  Threads: calls that change a cache (append, evict, reset,
 *     set_state, destroy) must not run at the same time as any other call on that
 *     cache; calls that take it as const (the attention calls, query, get_state,
 *     key_segments, export) may be issued by several host threads at once on one
 *     handle -- the G candidates of a group decoding against one shared prefix --
 *     each with its own stream and output buffers.
 *   - bf16 tensors Q, O, K_chunk, V_chunk, dO, dQ, dK_chunk, dV_chunk are
 *     contiguous [batch, tokens, heads, head_dim].  LSE and delta are fp32
 *     [batch, heads, tokens].  Data pointers must be 16-byte aligned.
 *   - Functions return ASTRO_OK or an error code; they never throw or exit, and
 *     on an error the cache metadata is unchanged and nothing was launched.
 */
#ifndef ASTRO_H_
#define ASTRO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct astro_kvcache astro_kvcache_t; /* opaque, host side */

typedef enum {
  ASTRO_OK = 0,
  ASTRO_ERR_NULL = 1,      /* a required pointer is null */
  ASTRO_ERR_SHAPE = 2,     /* unsupported or inconsistent shape (head_dim not 64/128, batch mismatch, empty key set) */
  ASTRO_ERR_ALIGN = 3,     /* a data pointer is not 16-byte aligned */
  ASTRO_ERR_CAPACITY = 4,  /* append would hold more than S+L frames, or a buffer is too small */
  ASTRO_ERR_UNDERFLOW = 5, /* evict asks for more window frames than are held */
  ASTRO_ERR_ARCH = 6,      /* current device is not compute capability 10.x */
  ASTRO_ERR_CUDA = 7,      /* a CUDA runtime/driver call failed */
  ASTRO_ERR_TIMEOUT = 8    /* a bounded device-side wait ran out (see astro_last_device_status) */
} astro_status_t;

typedef struct {
  int cache_batch;      /* B_c: samples with their own cache; 1 = one shared frozen prefix for a group */
  int heads;            /* H */
  int head_dim;         /* D: 64 or 128 */
  int tokens_per_frame; /* T */
  int sink_frames;      /* S >= 0 */
  int window_frames;    /* L >= 1: slots of the sliding window */
} astro_kvcache_desc_t;

/* Bytes the caller must allocate for K (and the same again for V):
 * B_c * H * (S+L) * T * D * 2.  Returns 0 for an invalid descriptor. */
size_t astro_kvcache_storage_bytes(const astro_kvcache_desc_t* desc);

/* Sec. 3.2, "Rolling KV Cache with Frame Sinks": bind caller-allocated device
 * storage for the restricted context C_n (S sink frames + window of L frames),
 * so that resident KV memory is constant however long the video grows.
 * k_storage/v_storage: device, >= bytes_each each, 16-byte aligned; the layout
 * inside is private ([B_c, H, slot, T, D]).  The storage need not be initialised.
 * The cache starts empty.  *out receives the handle.  The call also encodes the
 * tensor maps of the storage (a host-only driver call; nothing is launched). */
astro_status_t astro_kvcache_create(const astro_kvcache_desc_t* desc, void* k_storage, void* v_storage,
                                    size_t bytes_each, astro_kvcache_t** out);

/* Frees the host-side handle only. */
astro_status_t astro_kvcache_destroy(astro_kvcache_t* cache);

/* Empties the cache (the next S appended frames become the new sink); storage is kept. */
astro_status_t astro_kvcache_reset(astro_kvcache_t* cache);

/* Sec. 3.3, "Streaming Long Tuning" (the forward pass accumulates the KV cache up
 * to the target step) and Sec. 3.2: store K and V of n_frames new frames.
 * k, v: device bf16 [B_c, n_frames*T, H, D].  The first S frames ever appended
 * fill the sink; later ones take the next free window slot.  The copy is
 * bit-exact.  There is no implicit eviction: ASTRO_ERR_CAPACITY if the cache
 * would hold more than S+L frames. */
astro_status_t astro_kvcache_append(astro_kvcache_t* cache, const void* k, const void* v, int n_frames,
                                    void* stream);

/* Sec. 3.2: the window keeps "the L most recent frames": drop the n_frames
 * oldest window frames.  Sink frames are never dropped.  The window is a ring,
 * so this advances an index and moves no bytes (the stream is unused today).
 * ASTRO_ERR_UNDERFLOW if n_frames exceeds the window frames held. */
astro_status_t astro_kvcache_evict(astro_kvcache_t* cache, int n_frames, void* stream);

/* Host-side state: frames held in the sink, in the window, and frames appended
 * since create/reset.  Any of the three HOST pointers may be null. */
astro_status_t astro_kvcache_query(const astro_kvcache_t* cache, int* sink_held, int* window_held,
                                   int64_t* frames_seen);

/* Checkpoint / resume.  The cache's whole state is the caller's storage plus this small record: a caller
 * that saves both (Sec. 3.3: the forward roll that accumulates the cache is the expensive part of a
 * training step) can later bind the saved bytes to a new handle with astro_kvcache_create and restore the
 * record with astro_kvcache_set_state.  HOST pointers.  set_state returns ASTRO_ERR_SHAPE if the record
 * does not fit the descriptor (counts out of range, window frames without a full sink). */
typedef struct {
  int sink_held;       /* frames in the sink slots */
  int window_head;     /* ring index of the oldest window frame, 0..L-1 */
  int window_held;     /* frames in the window ring */
  int64_t frames_seen; /* frames appended since create/reset */
} astro_kvcache_state_t;
astro_status_t astro_kvcache_get_state(const astro_kvcache_t* cache, astro_kvcache_state_t* state);
astro_status_t astro_kvcache_set_state(astro_kvcache_t* cache, const astro_kvcache_state_t* state);

/* Inspection aid (host only, launches nothing): the physical token ranges of the cache storage that an
 * attention call would walk in the cache's present state -- at most two, merged where adjacent, because the
 * window ring can be split by its wrap-around or by a hole left by evict -- followed by the chunk's own keys
 * when n_kc > 0.  HOST arrays of at least 3 entries each: first token, token count, and 1 for the chunk
 * segment / 0 for a cache segment.  *n_segments receives the number of entries written. */
astro_status_t astro_kvcache_key_segments(const astro_kvcache_t* cache, int n_kc, int* n_segments, int* first_token,
                                          int* token_count, int* from_chunk);

/* Inspection aid: write the held frames in logical order (sink frames, then
 * window oldest to newest) to k_out, v_out: device bf16 [B_c, held*T, H, D]. */
astro_status_t astro_kvcache_export(const astro_kvcache_t* cache, void* k_out, void* v_out, void* stream);

/* Sec. 3.2 (while the next clip is generated, attention is restricted to the cached
 * keys and values of the context C_n; G candidates decode against one shared prefix)
 * -- forward of chunk attention.  For every sample b, head h and chunk query i:
 *   keys/values = every token held in the cache (of sample b, or of the single
 *   shared cache when B_c = 1) followed by the n_kc chunk tokens;
 *   s_ij = scale * q_i . k_j;  LSE_i = ln sum_j exp(s_ij);  o_i = sum_j exp(s_ij - LSE_i) v_j.
 * q [batch, n_q, H, D], k_chunk/v_chunk [batch, n_kc, H, D] (may be null when
 * n_kc = 0), o [batch, n_q, H, D] bf16, lse [batch, H, n_q] fp32 (may be null).
 * cache may be null (no context).  n_q, n_kc are token counts and need not be
 * multiples of T or of any tile.  ASTRO_ERR_SHAPE if there is no key at all,
 * batch differs from B_c and B_c != 1, or scale is negative or not finite.
 * bf16 products, fp32 accumulation and softmax. */
astro_status_t astro_chunk_attn_fwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                    const void* v_chunk, int batch, int heads, int head_dim, int n_q,
                                    int n_kc, float scale, void* o, float* lse, void* stream);

/* Scratch bytes astro_chunk_attn_bwd needs (delta, fp32 [batch, H, n_q], rounded up). */
size_t astro_chunk_attn_bwd_workspace_bytes(int batch, int heads, int n_q, int head_dim);

/* Sec. 3.3, "Streaming Long Tuning": the KV cache of all preceding frames is
 * detached; gradients flow through the active window only.  Given dO and the
 * forward's O and LSE:
 *   p_ij = exp(s_ij - LSE_i); dp_ij = dO_i . v_j; delta_i = dO_i . o_i;
 *   ds_ij = p_ij (dp_ij - delta_i);
 *   dq_i = scale * sum over ALL keys of ds_ij k_j;
 *   dk_j = scale * sum_i ds_ij q_i and dv_j = sum_i p_ij dO_i for CHUNK keys only.
 * dq [batch, n_q, H, D], dk_chunk/dv_chunk [batch, n_kc, H, D], all bf16 written
 * from fp32 accumulators (dk_chunk/dv_chunk may be null when n_kc = 0).
 * workspace: device scratch of at least astro_chunk_attn_bwd_workspace_bytes(). */
astro_status_t astro_chunk_attn_bwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                    const void* v_chunk, const void* o, const float* lse, const void* d_o,
                                    int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                    void* dq, void* dk_chunk, void* dv_chunk, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* The three stages of astro_chunk_attn_bwd as calls of their own (same layouts, same checks); the
 * composite call is exactly delta, then dq, then dkv on one stream.  A caller that trains only the
 * query side can skip the last stage.
 *   delta: delta[b,h,i] = sum_d dO[b,i,h,d] * O[b,i,h,d], fp32 [batch, H, n_q] (device, 16-byte aligned).
 *   dq:    dQ over ALL keys (cache + chunk) from Q, dO, LSE, delta.
 *   dkv:   dK, dV of the chunk's own keys from Q, dO, LSE, delta (no cache involved: context is detached). */
astro_status_t astro_chunk_attn_bwd_delta(const void* o, const void* d_o, int batch, int heads, int head_dim,
                                          int n_q, float* delta, void* stream);
astro_status_t astro_chunk_attn_bwd_dq(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                       const void* v_chunk, const float* lse, const float* delta, const void* d_o,
                                       int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                       void* dq, void* stream);
astro_status_t astro_chunk_attn_bwd_dkv(const void* q, const void* k_chunk, const void* v_chunk, const float* lse,
                                        const float* delta, const void* d_o, int batch, int heads, int head_dim,
                                        int n_q, int n_kc, float scale, void* dk_chunk, void* dv_chunk,
                                        void* stream);

/* Continue a cache as another one: empties `dst` and copies frames of `src` into it, as if they had been appended to it
 * in the order of `frames` (its first S_dst frames become the sink).  frames: HOST array of n_frames logical frame
 * indices of src (0 = oldest: sink frames, then the window oldest to newest; repeats allowed); null with
 * n_frames = -1 takes every held frame, n_frames = 0 none.  So the call copies, forks (one shared prefix, cache_batch 1, into one cache per
 * candidate), reorders and compacts.
 * parents: device int32 [dst cache_batch], the sample of src that each sample of dst continues; null: sample b
 * continues sample b, or sample 0 of a one-sample src.  A parent outside src leaves zeros in the copied frames.
 * dst's frames_seen becomes src's, or the number of copied frames where repeats make that larger (a cache has seen at least
 * the frames it holds).  ASTRO_ERR_SHAPE: other heads, head_dim or tokens_per_frame, caches of different kinds (16 and 8 bits); parents null and
 * cache batches that are neither equal nor 1; a frame index that src does not hold; storage of dst that overlaps src's.
 * ASTRO_ERR_CAPACITY: more frames than dst holds.  Calls on dst and src obey the rules of calls that change a cache
 * (dst) and of calls that take it as const (src). */
astro_status_t astro_kvcache_fork(astro_kvcache_t* dst, const astro_kvcache_t* src, const int32_t* parents,
                                  const int* frames, int n_frames, void* stream);

/* ---- rotary positions -------------------------------------------------------------------------------------------
 * The attention calls take Q and K with their positions already in them; this is the operator that puts them there.
 * A token has `axes` integer coordinates (1 for plain sequences; 3 for frame, row and column of a latent video).  The
 * first rot_dim elements of a head form rot_dim/2 pairs, dealt to the axes in order (axis_pairs[0] pairs turn with
 * coordinate 0, and so on); pair i of an axis with n pairs turns by f_i = base^(-i/n) radians per position.
 * Contexts longer than the trained one, for the axes in the bit mask scaled_axes:
 *   NONE    f_i
 *   LINEAR  f_i / factor
 *   BASE    base replaced by base * factor^(n/(n-1)): the fastest pair is left alone, the slowest divided by factor
 *   RAMP    with r = original_length f_i / 2 pi turns over the trained length and g = (r - ramp_low) /
 *           (ramp_high - ramp_low) clamped to [0, 1]:  f_i (g + (1 - g) / factor)
 * magnitude multiplies cosines and sines; 0 means 1, or 0.1 ln(factor) + 1 for RAMP.  ASTRO_ERR_SHAPE for a table whose
 * frequencies are not all positive finite doubles or whose magnitude is no positive finite float. */
typedef struct astro_rope astro_rope_t; /* opaque, host side, owns no device memory */
enum { ASTRO_ROPE_INTERLEAVED = 0, ASTRO_ROPE_HALVES = 1 };       /* pairs (2p, 2p+1) or (p, p + rot_dim/2) */
enum { ASTRO_ROPE_SCALE_NONE = 0, ASTRO_ROPE_SCALE_LINEAR = 1, ASTRO_ROPE_SCALE_BASE = 2, ASTRO_ROPE_SCALE_RAMP = 3 };
enum { ASTRO_BF16 = 0, ASTRO_F16 = 1, ASTRO_F32 = 2 };
typedef struct {
  int head_dim;        /* multiple of 8, 8..256 */
  int rot_dim;         /* even, 2..head_dim; the elements behind it are copied */
  int layout;
  int axes;            /* 1..4 */
  int axis_pairs[4];   /* each >= 1, sum = rot_dim / 2 */
  double base;         /* > 0 */
  int scaling;
  int scaled_axes;     /* bit a: axis a is scaled */
  double factor;       /* >= 1 */
  double original_length, ramp_low, ramp_high; /* RAMP only: > 0, ramp_low < ramp_high */
  double magnitude;    /* >= 0 */
} astro_rope_desc_t;
typedef struct {
  int64_t batch, token, head; /* strides in elements; the elements of a head are contiguous */
} astro_strides_t;

astro_status_t astro_rope_create(const astro_rope_desc_t* desc, astro_rope_t** out);
astro_status_t astro_rope_destroy(astro_rope_t* rope);
/* Inspection aid: radians per position of every pair (HOST, rot_dim/2 values) and the factor on cosines and sines. */
astro_status_t astro_rope_frequencies(const astro_rope_t* rope, double* frequencies, double* magnitude);
/* Rotates q [batch, n_tokens, heads_q, head_dim] and, unless null, k [batch, n_tokens, heads_k, head_dim] into q_out and
 * k_out.  inverse = 1 applies the transpose (rotates back, with the same magnitude): the gradient of the inputs from the
 * gradient of the outputs.  dtype: type of all four tensors; fp32 arithmetic, one rounding.
 * positions: device int32 [positions_batch, n_tokens, axes], positions_batch = batch or 1 (the same for every
 * sample); any int32 value, angles keep their accuracy to the far end of it.
 * in_strides (of q and k alike) and out_strides (of q_out and k_out): null = contiguous.  Pointers and strides must be
 * multiples of 16 bytes (ASTRO_ERR_ALIGN).  An input stride may be 0 (a broadcast input, whose gradient is the sum of the
 * copies' gradients: the caller's to take); outputs must not overlap themselves (ASTRO_ERR_SHAPE).  q_out = q (and k_out = k) rotates in place, with equal strides; otherwise outputs
 * must not overlap inputs.  n_tokens = 0 is an empty call. */
astro_status_t astro_rope_apply(const astro_rope_t* rope, int inverse, const void* q, const void* k,
                                const int32_t* positions, int positions_batch, int batch, int n_tokens, int heads_q,
                                int heads_k, int dtype, const astro_strides_t* in_strides, void* q_out, void* k_out,
                                const astro_strides_t* out_strides, void* stream);

/* Host only: what astro_rope_apply would answer to these arguments before it launches anything.  For callers that rotate q and
 * k in two calls (different strides) and want neither if one of them is refused. */
astro_status_t astro_rope_apply_check(const astro_rope_t* rope, int inverse, const void* q, const void* k,
                                      const int32_t* positions, int positions_batch, int batch, int n_tokens, int heads_q,
                                      int heads_k, int dtype, const astro_strides_t* in_strides, void* q_out, void* k_out,
                                      const astro_strides_t* out_strides);

/* ---- the cache in 8 bits ------------------------------------------------------------------------------------------
 * A rolling cache that takes 8 bits per element and 8 per row (the head_dim elements of one head and token): half the memory
 * of astro_kvcache_create's, so twice the frames or samples.  A row x is held as
 *   e = the smallest whole number with max |x_d| <= 448 * 2^e over the row's finite elements, -124 at least, and
 *   e4m3(x_d * 2^-e) for every element, rounded to nearest even; an infinity or NaN becomes NaN, the others are not touched by it.
 * (Elements of 248 * 2^120 and more, which would round beyond the largest float, are held as 240 * 2^120.)
 * What it stands for, e4m3 value times 2^e, is a bf16 number exactly: reading it back in bf16 or fp32 rounds nothing.
 * The handle is an astro_kvcache_t: destroy, reset, evict, query, get_state, set_state, key_segments, export, append (which takes
 * bf16) and fork (from one such cache into another) do for it what they do for the other kind.  The calls that read a 16-bit
 * cache's rows (astro_chunk_attn_*, astro_block_pool, astro_block_select, astro_sparse_attn_*) answer ASTRO_ERR_SHAPE to
 * it, and the calls below to a 16-bit one. */
/* Bytes for K (and the same again for V); 0 for an invalid descriptor. */
size_t astro_kvcache8_storage_bytes(const astro_kvcache_desc_t* desc);
/* As astro_kvcache_create; the layout inside the storage is private. */
astro_status_t astro_kvcache8_create(const astro_kvcache_desc_t* desc, void* k_storage, void* v_storage, size_t bytes_each,
                                     astro_kvcache_t** out);
/* As astro_kvcache_append, the rows being quantised on the way.  k, v: device [B_c, n_frames * T, H, D] of type dtype, strides
 * (of both, null = contiguous) and pointers multiples of 16 bytes. */
astro_status_t astro_kvcache8_append(astro_kvcache_t* cache, const void* k, const void* v, int n_frames, int dtype,
                                     const astro_strides_t* strides, void* stream);
/* What the n_frames held frames from logical frame first_frame on stand for, in logical order: k_out, v_out device
 * [B_c, n_frames * T, H, D], contiguous, of type dtype (in fp16 values are rounded, and infinite beyond its range).
 * n_frames = 0 is an empty call. */
astro_status_t astro_kvcache8_read(const astro_kvcache_t* cache, int first_frame, int n_frames, int dtype, void* k_out, void* v_out,
                                   void* stream);

/* astro_chunk_attn_fwd over a cache in 8 bits: the keys and values of the cached tokens are what their rows stand for, the
 * chunk's are bf16.  Same layouts, results and errors; cache may be null.  workspace: device scratch, 16-byte aligned, at least
 * astro_chunk_attn8_fwd_workspace_bytes() for the frames that the cache holds at the time of the call (it may be null where that is 0).  Many
 * queries: the held rows in bf16; few: the parts of lists that several CTAs share.  With few queries a cached key counts as zero in O where its
 * weight times the power of two of its value row is below 2^-120 of the query's largest such product, and an element of q has fewer
 * bits below 2^-31 of its row's largest and counts as zero below 2^-38 (for the cached keys). */
size_t astro_chunk_attn8_fwd_workspace_bytes(const astro_kvcache_t* cache, int batch, int heads, int head_dim, int n_q, int n_kc);
astro_status_t astro_chunk_attn8_fwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk, int batch,
                                     int heads, int head_dim, int n_q, int n_kc, float scale, void* o, float* lse, void* workspace,
                                     size_t workspace_bytes, void* stream);
/* astro_chunk_attn_bwd over a cache in 8 bits, the cached context detached: dQ over all keys, dK and dV of the chunk's own.  Over one
 * key in all dQ and dK are zeros.  workspace: as for the forward, astro_chunk_attn8_bwd_workspace_bytes().  All sums have one fixed
 * order: the same call gives the same bits. */
size_t astro_chunk_attn8_bwd_workspace_bytes(const astro_kvcache_t* cache, int batch, int heads, int head_dim, int n_q, int n_kc);
astro_status_t astro_chunk_attn8_bwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk,
                                     const void* o, const float* lse, const void* d_o, int batch, int heads, int head_dim, int n_q,
                                     int n_kc, float scale, void* dq, void* dk_chunk, void* dv_chunk, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* ---- attention over chosen key blocks ---------------------------------------------------------------------------
 * The keys of a call are cut into blocks of block_tokens tokens (a multiple of 8, 8..128): every held cache frame, in
 * logical order, into ceil(T / block_tokens) blocks, then the chunk's n_kc tokens into ceil(n_kc / block_tokens).
 * The last block of a frame and of the chunk may be shorter.  Blocks are numbered in that order, from 0.
 * ASTRO_QUERY_BLOCK neighbouring queries share one list of key blocks; a query block that is shorter (the last one,
 * or a single query) has its list to itself. */
#define ASTRO_QUERY_BLOCK 128
/* Longest list of a query block (n_select): the bounded waits inside the kernels are laid out for lists of that length. */
#define ASTRO_MAX_SELECT 65536
/* Host only: number of cache blocks and of chunk blocks (HOST pointers, either may be null). */
astro_status_t astro_block_count(const astro_kvcache_t* cache, int n_kc, int block_tokens, int* ctx_blocks,
                                 int* chunk_blocks);

/* Means of the keys of cache blocks: for the n_frames held frames from logical frame first_frame on,
 * pooled[b, h, slot, i, :] = mean over the tokens of block i of the frame's keys, fp32 from fp64 sums.
 * pooled: device fp32 [B_c, H, S+L, ceil(T / block_tokens), D], indexed by storage slot, so an evict or an append
 * leaves the means of the other frames valid: a caller pools new frames once, when they are appended. */
astro_status_t astro_block_pool(const astro_kvcache_t* cache, int first_frame, int n_frames, int block_tokens,
                                float* pooled, void* stream);

/* Chooses key blocks: score(i, j) = (mean of the queries of query block i) . (mean of the keys of block j), means in
 * fp32, products and sums in fp64.  blocks: device int32 [batch, H, ceil(n_q / ASTRO_QUERY_BLOCK), n_select] receives
 * the n_select blocks of the highest scores in ascending order, with -1 behind them if there are fewer blocks.  Equal
 * scores go to the lower block; NaN ranks below every number.  keep: blocks that come before every other one
 * whatever their score (the lower ones first), ASTRO_KEEP_SINK those of the sink frames, ASTRO_KEEP_CHUNK the chunk's.
 * pooled: the means of every held frame (may be null if the cache is null or empty); k_chunk null when n_kc = 0.
 * workspace: device scratch, 16-byte aligned, at least astro_block_select_workspace_bytes().  Like every workspace here it
 * is written and read by the call's kernels only: calls that may overlap on the GPU (other streams, replayed graphs) need
 * one each.
 * ASTRO_ERR_SHAPE as for the attention calls, for more than ASTRO_SELECT_MAX_BLOCKS blocks and for an n_select outside
 * 1..ASTRO_MAX_SELECT. */
#define ASTRO_SELECT_MAX_BLOCKS 24576
enum { ASTRO_KEEP_SINK = 1, ASTRO_KEEP_CHUNK = 2 };
size_t astro_block_select_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_kc, int block_tokens);
astro_status_t astro_block_select(const astro_kvcache_t* cache, const float* pooled, const void* q, const void* k_chunk,
                                  int batch, int heads, int head_dim, int n_q, int n_kc, int block_tokens, int n_select,
                                  int keep, int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream);

/* Forward of attention over chosen key blocks: astro_chunk_attn_fwd with the keys of query block i restricted to the
 * blocks that its list names.  blocks: device int32 [batch, H, ceil(n_q / ASTRO_QUERY_BLOCK), n_select] in any order.  An
 * entry outside [0, number of blocks) names none; a block named twice counts twice.  A query with no key (an empty list) gets
 * O = 0 and LSE = -infinity.  The other arguments, layouts and errors are astro_chunk_attn_fwd's; n_select is 1..ASTRO_MAX_SELECT.
 * workspace: device scratch, 16-byte aligned, at least astro_sparse_attn_fwd_workspace_bytes() (0 for all but a few
 * queries: their lists are cut into ranges that run side by side; then it may be null). */
size_t astro_sparse_attn_fwd_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_select, int block_tokens);
astro_status_t astro_sparse_attn_fwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk,
                                     const int32_t* blocks, int n_select, int block_tokens, int batch, int heads,
                                     int head_dim, int n_q, int n_kc, float scale, void* o, float* lse, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* Its backward, the cached context detached as in astro_chunk_attn_bwd: from dO and the forward's O and LSE (same lists),
 * dQ over the listed keys, dK and dV of the chunk's own tokens.  A query without a key has dQ = 0; a chunk block that no
 * list names has dK = dV = 0; a block named twice counts twice here too.  All sums have one fixed order: the same call
 * gives the same bits.  Other arguments as for astro_chunk_attn_bwd; workspace: device scratch, 16-byte aligned, at least
 * astro_sparse_attn_bwd_workspace_bytes(). */
size_t astro_sparse_attn_bwd_workspace_bytes(int batch, int heads, int head_dim, int n_q, int n_kc, int n_select,
                                             int block_tokens);
astro_status_t astro_sparse_attn_bwd(const astro_kvcache_t* cache, const void* q, const void* k_chunk, const void* v_chunk,
                                     const int32_t* blocks, int n_select, int block_tokens, const void* o, const float* lse,
                                     const void* d_o, int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                     void* dq, void* dk_chunk, void* dv_chunk, void* workspace, size_t workspace_bytes,
                                     void* stream);

/* ---- sliding window with sinks over whole sequences ---------------------------------------------------------------
 * The attention of the streaming scheme for all the blocks of a sequence at once, as it is trained or as a prompt is taken in:
 * with c = i / block_tokens, query i sees key j iff
 *     j < min(len, (c + 1) * block_tokens)  and  (j < sink_tokens or j >= (c + 1) * block_tokens - window_tokens),
 * its own block whole, the window_tokens - block_tokens tokens in front of it, and the sink.  (A cache of S + L frames from which a caller
 * evicts down to S + L - c frames before every chunk of c frames of T tokens shows a chunk the same keys with block_tokens = c T,
 * sink_tokens = S T, window_tokens = L T.)  block_tokens = 1 is the sliding window of single tokens; a window_tokens of n_tokens +
 * block_tokens and more shows every token in front.  heads / kv_heads neighbouring heads share a head of k and v.
 *   q, o [batch, n_tokens, heads, head_dim], k, v [batch, n_tokens, kv_heads, head_dim], bf16, LSE fp32 [batch, heads, n_tokens].
 *   q_strides, k_strides, v_strides: null = contiguous; multiples of 16 bytes, no stride of 0.  o is contiguous.
 *   lengths: device int32 [batch], tokens of each sample (values outside 0..n_tokens count as the nearer end); null: n_tokens each.  What k, v and q
 *   hold from there on does not matter, NaN included; those queries get O = 0 and LSE = -infinity.
 * A NaN or infinity reaches the queries that see it and no others (a tile of 128 queries that is met by one goes key by key, which
 * is slow).  lse may be null.  o must not overlap q, k or v.  n_tokens = 0 is an empty call.
 * ASTRO_ERR_SHAPE: head_dim not 64 or 128, heads not a multiple of kv_heads, window_tokens < block_tokens, n_tokens > 2^29, a scale that
 * is negative or not finite.  bf16 products, fp32 accumulation and softmax. */
typedef struct {
  int batch, n_tokens, heads, kv_heads, head_dim;
  int block_tokens, window_tokens, sink_tokens;
} astro_window_desc_t;
astro_status_t astro_window_attn_fwd(const astro_window_desc_t* desc, const void* q, const astro_strides_t* q_strides, const void* k,
                                     const astro_strides_t* k_strides, const void* v, const astro_strides_t* v_strides,
                                     const int32_t* lengths, float scale, void* o, float* lse, void* stream);
/* Its backward, nothing detached: dQ, and dK and dV of every token, summed over the heads that share it, from dO and the forward's
 * O and LSE (all contiguous, as are dq, dk and dv).  Queries and keys from a sequence's length on get zeros, and what o, lse and d_o
 * hold there does not matter.  A query that sees one key has dQ = 0.  Outputs must not overlap inputs.  workspace: device scratch, 16-byte aligned, at least astro_window_attn_bwd_workspace_bytes().  All sums have one
 * fixed order: the same call gives the same bits. */
size_t astro_window_attn_bwd_workspace_bytes(int batch, int heads, int n_tokens, int head_dim);
astro_status_t astro_window_attn_bwd(const astro_window_desc_t* desc, const void* q, const astro_strides_t* q_strides, const void* k,
                                     const astro_strides_t* k_strides, const void* v, const astro_strides_t* v_strides,
                                     const int32_t* lengths, const void* o, const float* lse, const void* d_o, float scale, void* dq,
                                     void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream);

/* Eq. 1, Eq. 2 and the selective KL term of Sec. 3.4 (Algorithm 2, "Policy loss on window"), fused with
 * the gradient for the current policy, over the velocity tensors of the active window:
 *   v+ = (1-beta) v_old + beta v_theta;  v- = (1+beta) v_old - beta v_theta;
 *   policy_i = r_i ||v+ - target||^2 + (1 - r_i) ||v- - target||^2;   kl_i = ||v_theta - v_ref||^2
 * per sample i, with ||.||^2 the plain sum of squares over the sample's `elems` elements, and
 *   grad = d/d v_theta of sum_i (w_policy_i policy_i + w_kl_i kl_i)
 * (the caller folds 1/elems, 1/batch, lambda_KL, the uncertainty mask and 1/|M| into the weights).
 * v_theta, v_old, v_ref, v_target, grad: device bf16 [batch, elems], 16-byte aligned, elems a multiple of 8.
 * r_tilde, w_policy, w_kl, policy_out, kl_out: device fp32 [batch].  v_ref and kl_out may be null together
 * (no KL term); w_policy null means 1, w_kl null means 0; grad may be null (losses only).  policy_out and
 * kl_out are overwritten.  fp32 arithmetic; the per-sample sums use atomics, so their last bits depend on
 * the order of the blocks. */
astro_status_t astro_nft_loss(const void* v_theta, const void* v_old, const void* v_ref, const void* v_target,
                              const float* r_tilde, const float* w_policy, const float* w_kl, int batch,
                              long long elems, float beta, float* policy_out, float* kl_out, void* grad,
                              void* stream);

/* The paper has no counterpart for this call: it exists for callers that must not allocate device
 * memory around the backward -- a training loop whose allocator is frozen after warm-up, a plug-in
 * that runs inside someone else's memory pool, a host thread that may not take the allocator's lock.
 * Such callers cannot provide the delta scratch that astro_chunk_attn_bwd asks for, so this variant
 * keeps it in a fixed device array inside the library instead: ASTRO_BWD_STATIC_MAX_ROWS fp32 values
 * (1 MiB), resident on every GPU that loads the library until the process exits.
 * Same inputs, outputs, layouts and results as astro_chunk_attn_bwd, without the workspace arguments.
 * It calls no cudaMalloc/cudaFree and no allocating library routine.
 *   - ASTRO_ERR_CAPACITY if batch * heads * n_q exceeds ASTRO_BWD_STATIC_MAX_ROWS; nothing is launched.
 *   - The first call on each device looks up the array's device address (with that device current);
 *     make that first call outside any stream capture.
 *   - All calls on a device share the one array: two calls whose kernels may overlap on the GPU
 *     (different streams, no ordering between them) race on it.  Calls on one stream are safe.  The
 *     array keeps the previous call's delta; every element a call reads it has written first. */
#define ASTRO_BWD_STATIC_MAX_ROWS 262144
astro_status_t astro_chunk_attn_bwd_static(const astro_kvcache_t* cache, const void* q, const void* k_chunk,
                                           const void* v_chunk, const void* o, const float* lse, const void* d_o,
                                           int batch, int heads, int head_dim, int n_q, int n_kc, float scale,
                                           void* dq, void* dk_chunk, void* dv_chunk, void* stream);

/* Every device-side wait in the kernels is bounded; one that runs out records a
 * code in a device status word instead of hanging.  This call synchronises the
 * current device, reads and clears that word: ASTRO_OK, or ASTRO_ERR_TIMEOUT
 * (then *detail, a HOST pointer that may be null, receives the raw word). */
astro_status_t astro_last_device_status(uint32_t* detail);

/* Self-test of that mechanism (the paper has no counterpart): enqueues a one-warp kernel that waits about a
 * millisecond on a barrier nothing will ever complete.  The kernel gives up, ends normally and leaves the
 * time-out in the status word, so the next astro_last_device_status returns ASTRO_ERR_TIMEOUT and the
 * context stays usable.  Nothing faults or hangs.  The wait runs out for one lane of the warp only: were the others to go
 * on without it, bit 1 of the raw word would be set as well. */
astro_status_t astro_selftest_wait_timeout(void* stream);

/* Diagnostic switch (the paper has no counterpart).  The forward kernel first runs a fast pass in which a
 * query row keeps the maximum of its first key tile as its one reference exponent, and repeats a 128-query
 * tile with a running reference (the "safe pass") only if a row sum left the range fp32 can hold.
 *   mode 0  normal operation;
 *   mode 1  every later astro_chunk_attn_fwd of this process runs the safe pass only (astro_sparse_attn_fwd likewise its
 *           own pass with a running reference);
 *   mode 2  head_dim 128 calls run the CTA-pair kernel (two query tiles share every K/V tile through one
 *           tcgen05 cta_group::2 MMA); it has no safe pass of its own: a call whose rows would need one leaves
 *           a flag that astro_debug_pair_flag reads (and clears) after synchronising the device.
 * Results agree within the rounding of bf16 in every mode; the switch exists so that tests and benchmarks can
 * reach each code path on ordinary inputs.  Process-wide, not stream-ordered: it applies to calls made after it
 * returns.  ASTRO_ERR_SHAPE for any other mode. */
astro_status_t astro_debug_forward_mode(int mode);
astro_status_t astro_debug_pair_flag(int* flag);

/* Static, never null. */
const char* astro_status_string(astro_status_t status);

#ifdef __cplusplus
}
#endif
#endif /* ASTRO_H_ */
