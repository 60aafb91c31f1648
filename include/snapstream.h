/*
 * snapstream.h -- C ABI of the SnapStream hot path on MI355X (gfx950).
 *
 * SnapStream (arXiv 2511.03092) keeps, per sequence and KV head, a cache of
 * fixed size B = sink + recent + topk rows (Sec. III-A):
 *   rows [0, sink)                 attention-sink tokens (StreamingLLM),
 *   rows [sink, sink+recent)       the rolling window of recent tokens, kept as
 *                                  a ring buffer (Sec. III-B.1),
 *   rows [sink+recent, B)          the top-K tokens chosen by SnapKV at the end
 *                                  of prefill (Sec. III-B.2, Eq. 1-3), followed
 *                                  by zeroed padding rows when fewer exist.
 * The library fills that cache from a padded prefill (snap_compress; or
 * snap_prefill, which also computes the prompt's causal attention and takes
 * the window statistics from it), writes
 * each decoded token into its ring row (snap_cache_append, Sec. III-C), and
 * runs decode attention over the valid rows (snap_decode_attn; snap_decode_step
 * does both for one layer).  Beside it stand rotary positions for the queries
 * and keys that go in (snap_rope) and a paged cache of growing length, for
 * layers that are not compressed and for sequences that are cut back to the
 * budget later by the attention their rows received (snap_paged_*).  The pages
 * themselves are handed out and taken back on the device (snap_pages_*), and a
 * cache that drops nothing holds its rows in blocks, in 8 bits with a scale for
 * each block and head, and may read only the blocks that matter to a query
 * (snap_block_*).
 *
 * Conventions shared by every call
 *  - Token positions are 0-based; a prompt of length L holds tokens 0..L-1 and
 *    the first decoded token is at position L.
 *  - Every pointer argument named as a tensor is DEVICE memory owned by the
 *    caller.  The library allocates nothing, frees nothing and never
 *    synchronises; all work is enqueued on `stream` (a hipStream_t, NULL = the
 *    null stream) and the call returns once it is launched.
 *  - Arguments are validated on the host before anything is launched; a
 *    failure returns a non-zero snap_status, launches nothing and leaves a
 *    message for snap_last_error().  A failed launch returns SNAP_ERR_HIP.
 *  - Per-sequence lengths and positions are device data, so a decode step
 *    needs no host round trip.  Device data out of range is handled without
 *    faulting: lengths are clamped to [0, max_len]; a slot id outside
 *    [0, n_slots) makes the call skip that sequence.
 *  - Inputs must not alias the cache.  Calls on disjoint buffers may run
 *    concurrently on different streams.  One exception to disjointness:
 *    snap_compress / snap_prefill calls of different layers for the same
 *    prompt may run concurrently although they share that slot's pos and
 *    n_topk entries, since those calls only write them, with the same values
 *    (L and min(K, |C|)).
 *  - Batch limits of the launch grids: n_seq * n_kv_heads <= 65535
 *    (snap_compress, snap_prefill, snap_prefill_attn, snap_paged_append,
 *    snap_paged_evict, snap_block_append) and n * n_q_heads <= 65535
 *    (snap_decode_attn, snap_decode_step, snap_paged_decode_attn,
 *    snap_paged_decode_step, snap_block_decode_attn, snap_block_decode_step);
 *    larger calls return SNAP_ERR_UNSUPPORTED (split the batch).
 */
#ifndef SNAPSTREAM_H
#define SNAPSTREAM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SNAP_OK = 0,
  SNAP_ERR_INVALID_ARG = 1, /* a parameter, pointer or size is invalid     */
  SNAP_ERR_UNSUPPORTED = 2, /* valid, but no kernel for this combination   */
  SNAP_ERR_WORKSPACE = 3,   /* workspace NULL or smaller than the query    */
  SNAP_ERR_HIP = 4          /* the HIP runtime reported an error on launch */
} snap_status;

typedef enum {
  SNAP_F32 = 0,
  SNAP_BF16 = 1,
  SNAP_FP8_E4M3 = 2, /* OCP E4M3 (fn): bias 7, max 448, no inf; cache only */
  SNAP_INT8 = 3      /* whole numbers -127..127; block caches only          */
} snap_dtype;

typedef enum {
  SNAP_POOL_MAX = 0, /* max pooling of the summed attention            */
  SNAP_POOL_AVG = 1  /* average pooling (Eq. 2), zero padding, / kernel */
} snap_pool;

typedef enum {
  SNAP_NORM_CAND = 0, /* softmax over the eviction candidates only (Eq. 3) */
  SNAP_NORM_ROW = 1   /* softmax over the whole causal row [0, i]          */
} snap_norm;

/* Who sets an fp8 cache's per-(slot, KV head) scales. */
typedef enum {
  SNAP_FP8_SCALES_GIVEN = 0, /* the caller, before compress / append           */
  SNAP_FP8_SCALES_AMAX = 1   /* snap_compress: amax / 448 over the rows the
                                compressed cache keeps (sinks, ring, selected;
                                1 when they are all zero), for K and V apart;
                                tokens appended later saturate at +-448 codes */
} snap_fp8_scales;

/* How decode reads the cache rows: a load hint.  Results agree to rounding
 * (under streaming loads the bf16 GQA kernel adds the dot products' 8-element
 * pieces in another order; the other kernels give the same bits). */
typedef enum {
  SNAP_KV_AUTO = 0,   /* streaming when the call's cache rows at the full
                         budget reach 128 MiB, cached loads otherwise          */
  SNAP_KV_STREAM = 1, /* non-temporal loads: the rows will not be read again
                         before the last-level cache (256 MB) has turned over,
                         e.g. many layers or large batches between two reads  */
  SNAP_KV_KEEP = 2    /* ordinary loads: the cache fits in the last-level cache
                         and is read again soon (a one-layer model, a small
                         batch)                                                 */
} snap_kv_reuse;

/* The method's hyper-parameters (Sec. III, Table 6's names). */
typedef struct {
  int32_t n_q_heads;   /* query heads; a multiple of n_kv_heads                 */
  int32_t n_kv_heads;  /* KV heads (1 for a shared latent cache)                */
  int32_t d_qk;        /* query/key width: 64, 128 or 576                        */
  int32_t d_v;         /* value width: 64, 128 or 512                            */
  int32_t v_in_k;      /* 1: latent cache (Sec. VI) -- one stored row per token
                          of width d_qk whose first d_v dims are the value; there
                          is no separate V input or V cache                       */
  int32_t sink;        /* L_sink >= 0                                            */
  int32_t recent;      /* L_recent >= 1 (ring length)                            */
  int32_t topk;        /* K >= 0                                                 */
  int32_t obs_window;  /* L_obs >= 1: queries of the last L_obs prompt tokens    */
  int32_t pool_kernel; /* odd, 1..63                                             */
  int32_t pool;        /* snap_pool                                              */
  int32_t norm;        /* snap_norm                                              */
  int32_t in_dtype;    /* q / k / v inputs: SNAP_F32 or SNAP_BF16                */
  int32_t kv_dtype;    /* cache storage: SNAP_F32, SNAP_BF16 (in_dtype == the
                          same) or SNAP_FP8_E4M3 (with SNAP_BF16 inputs)          */
  float sm_scale;      /* softmax scale; <= 0 means 1/sqrt(d_qk); a positive
                          value must be finite and at least 1e-30                */
  int32_t fp8_scales;  /* snap_fp8_scales (fp8 caches; ignored otherwise)        */
  int32_t fp8_qk;      /* decode attention over an fp8 cache: 0 = Q K^T in bf16
                          (the codes converted exactly); 1 = the query of each
                          head quantised to E4M3 with scale amax|q_h| / 448 (1
                          when q_h is zero; codes round to nearest even on the
                          fp32 quotient) and Q K^T on the fp8 MFMA.  Mode 1
                          changes the logits by the query's quantisation error
                          (about 2^-4 relative per element): it needs bf16
                          inputs, a GQA fp8 cache, d_qk = d_v = 128
                          (SNAP_ERR_UNSUPPORTED otherwise).  Values stay bf16
                          products.                                              */
  int32_t kv_reuse;    /* snap_kv_reuse: the decode kernels' load hint          */
} snap_params;

/* One layer's compressed cache (device memory, caller-owned, row-major):
 *   k       [n_slots][n_kv_heads][B][d_qk]  kv_dtype
 *   v       [n_slots][n_kv_heads][B][d_v]   kv_dtype; NULL when v_in_k
 *   k_scale [n_slots][n_kv_heads] fp32      FP8 only: stored code * scale is
 *   v_scale [n_slots][n_kv_heads] fp32      the value; set by the caller before
 *                                           compress/append, or by compress
 *                                           (fp8_scales); NULL otherwise. */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int32_t n_slots;
} snap_cache;

/* Slot metadata, shared by every layer (device int32[n_slots], caller-owned):
 *   pos[slot]    position of the token being decoded (L right after compress)
 *   n_topk[slot] real rows in the top-K region, min(max(L-sink-recent,0), K) */

/* Bytes of workspace snap_compress needs for n_seq sequences padded to
 * max_len.  0 on invalid parameters. */
size_t snap_compress_workspace(const snap_params* p, int32_t n_seq, int32_t max_len);

/* Bytes of workspace snap_decode_attn needs for n sequences.  0 on invalid
 * parameters. */
size_t snap_decode_workspace(const snap_params* p, int32_t n);

/* Compression at the end of prefill (Sec. III-B; Eq. 1-3).  For every
 * sequence b and KV head g:
 *   1. window scores: the G = n_q_heads/n_kv_heads query heads of group g at
 *      the last w_e = min(obs_window, L) positions score every key of the
 *      normaliser domain; softmax with sm_scale (Eq. 3);
 *   2. the softmax weights on the candidates C = [sink, L-recent) are summed
 *      over the window rows and the group's heads (Eq. 1);
 *   3. 1-D pooling (stride 1, pad pool_kernel/2) over C (Eq. 2);
 *   4. the min(K, |C|) candidates with the largest pooled score are kept (ties
 *      to the lower token index), in ascending token order;
 *   5. the cache of slot slot_ids[b] is rewritten: sinks, the last `recent`
 *      tokens at their ring rows (token t at row t < sink ? t :
 *      sink + (t - sink) mod recent), the kept tokens at rows sink+recent+m,
 *      zeros elsewhere (fp8: quantised with the slot/head scale), and
 *      pos[slot] = L, n_topk[slot] = min(K, |C|).
 * Arguments (device unless noted):
 *   slot_ids [n_seq] int32, lengths [n_seq] int32 (prompt lengths L),
 *   max_len (host) padded length of the inputs,
 *   q_obs [n_seq][n_q_heads][obs_window][d_qk] in_dtype; row obs_window-1 is
 *         position L-1 (rows before position 0 are ignored),
 *   k     [n_seq][n_kv_heads][max_len][d_qk] in_dtype (rows >= L never read),
 *   v     [n_seq][n_kv_heads][max_len][d_v]  in_dtype, NULL when v_in_k,
 *   sel_out    optional [n_seq][n_kv_heads][topk] int32: kept token indices,
 *              ascending, -1 padded (NULL to skip),
 *   pooled_out optional [n_seq][n_kv_heads][max_len] fp32: the pooled score of
 *              every candidate at its token index, NaN elsewhere (debug),
 *   workspace  >= snap_compress_workspace(p, n_seq, max_len) bytes, 256-byte
 *              aligned; its contents on entry do not matter.
 * n_seq == 0 is a no-op.  The sequences must target distinct slots. */
snap_status snap_compress(const snap_params* p, const snap_cache* cache, int32_t* pos,
                          int32_t* n_topk, int32_t n_seq, const int32_t* slot_ids,
                          const int32_t* lengths, int32_t max_len, const void* q_obs,
                          const void* k, const void* v, int32_t* sel_out, float* pooled_out,
                          void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace snap_prefill needs for n_seq sequences padded to
 * max_len: the snap_compress workspace, the window queries and a transposed
 * copy of V.  0 on invalid parameters. */
size_t snap_prefill_workspace(const snap_params* p, int32_t n_seq, int32_t max_len);

/* Prefill attention and compression in one call (Sec. IV-A's attention step
 * followed by Sec. III-B, with the window scores' softmax statistics taken
 * from the attention pass instead of a separate recompute, Sec. III-B.2).
 *   1. out[b][h][i] = sum_{j <= i} softmax_j(sm_scale q[b][h][i].k[b][g][j])
 *      v[b][g][j] for every position i < L (g = h / G), in bf16;
 *   2. the compression of snap_compress with q_obs = the queries of the last
 *      obs_window positions of q (same cache, pos, n_topk, sel_out and
 *      pooled_out results).
 * Arguments as snap_compress, except (device):
 *   q   [n_seq][n_q_heads][max_len][d_qk] bf16 (rows >= L never read),
 *   k   [n_seq][n_kv_heads][max_len][d_qk] bf16,
 *   v   [n_seq][n_kv_heads][max_len][d_v]  bf16,
 *   out [n_seq][n_q_heads][max_len][d_v]   bf16; rows >= L are not written,
 *   workspace >= snap_prefill_workspace(p, n_seq, max_len) bytes, 256-byte
 *             aligned; its contents on entry do not matter.
 * Supported: in_dtype bf16, d_qk == d_v in {64, 128} (v_in_k = 0), and
 * G = n_q_heads / n_kv_heads in {1, 2, 4, 8, 16}; SNAP_ERR_UNSUPPORTED otherwise.
 * out must not alias q, k or v.  n_seq == 0 is a no-op. */
snap_status snap_prefill(const snap_params* p, const snap_cache* cache, int32_t* pos, int32_t* n_topk,
                         int32_t n_seq, const int32_t* slot_ids, const int32_t* lengths, int32_t max_len,
                         const void* q, const void* k, const void* v, void* out, int32_t* sel_out,
                         float* pooled_out, void* workspace, size_t ws_bytes, void* stream);

/* The attention step of snap_prefill alone (Sec. IV-A): out as in
 * snap_prefill, no cache or metadata written, no selection.  For layers that
 * are not compressed, and for timing the attention apart from the
 * compression.  Same supported shapes, workspace (snap_prefill_workspace) and
 * errors as snap_prefill. */
snap_status snap_prefill_attn(const snap_params* p, int32_t n_seq, const int32_t* lengths, int32_t max_len,
                              const void* q, const void* k, const void* v, void* out, void* workspace,
                              size_t ws_bytes, void* stream);

/* Decode KV update (Sec. III-C): for each of the n sequences, the new token's
 * keys/values k_new [n][n_kv_heads][d_qk] and v_new [n][n_kv_heads][d_v]
 * (in_dtype; v_new NULL when v_in_k) are written to row
 * slot_of(pos[slot]) = pos < sink ? pos : sink + (pos - sink) mod recent,
 * which for pos >= sink is the paper's (pos - sink + recent) mod recent + sink.
 * Sequences with pos[slot] < 0 are skipped. */
snap_status snap_cache_append(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                              int32_t n, const int32_t* slot_ids, const void* k_new,
                              const void* v_new, void* stream);

/* Decode attention over the compressed cache (Sec. III-C; padding rows masked
 * per Sec. III-B.2).  For sequence b with p = pos[slot] (the token already
 * appended) the valid rows are [0, min(p+1, sink+recent)) and
 * [sink+recent, sink+recent+n_topk[slot]); each query head h attends its KV
 * head h / G: out[b][h] = sum_j softmax_j(sm_scale q.k_j) v_j.
 *   q   [n][n_q_heads][d_qk] in_dtype,
 *   out [n][n_q_heads][d_v]  out_dtype (SNAP_F32 or SNAP_BF16, rounded to
 *                            nearest even),
 *   workspace >= snap_decode_workspace(p, n) bytes, 256-byte aligned.
 * Rows outside the valid set are never read. */
snap_status snap_decode_attn(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                             const int32_t* n_topk, int32_t n, const int32_t* slot_ids,
                             const void* q, void* out, int32_t out_dtype, void* workspace,
                             size_t ws_bytes, void* stream);

/* One layer's decode step (Sec. III-C): snap_cache_append(k_new, v_new)
 * followed by snap_decode_attn, with the same arguments, results and cache
 * contents as those two calls on the same stream.  For bf16 and fp8 caches of
 * 64- and 128-wide rows and latent (576 / 512) caches of one KV head both
 * happen in one launch (the new token's row is read from k_new / v_new by the
 * workgroup that attends it, quantised there for an fp8 cache, and stored into
 * the cache in the same launch); other caches run the two launches.  The same
 * workspace as snap_decode_attn; k_new / v_new must not alias the cache. */
snap_status snap_decode_step(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                             const int32_t* n_topk, int32_t n, const int32_t* slot_ids,
                             const void* q, const void* k_new, const void* v_new, void* out,
                             int32_t out_dtype, void* workspace, size_t ws_bytes, void* stream);

/* Device memory of snap_decode_step_noalloc: one array of this many bytes per
 * GPU, owned by the library. */
#define SNAP_NOALLOC_SCRATCH_BYTES (32u << 20)

/* snap_decode_step for callers that cannot allocate device memory (code under
 * HIP graph capture that must not allocate, tight serving loops, harnesses
 * that forbid allocation): the same arguments, results and cache contents,
 * without the workspace.  The split-K partials go to a library-owned device
 * array of SNAP_NOALLOC_SCRATCH_BYTES per GPU (reserved with the library's
 * device code on the first call on that GPU, held until the process ends;
 * the call itself allocates nothing).  A call that would need more than that
 * (snap_decode_workspace(p, n) > SNAP_NOALLOC_SCRATCH_BYTES) returns
 * SNAP_ERR_WORKSPACE and launches nothing.  Every call on one GPU shares that
 * GPU's array: calls that may overlap in time on one GPU (other streams, or
 * other threads without ordering between them) race and give wrong results,
 * so serialise them.  What one call leaves in the array does not affect the
 * next (a call writes every byte it reads first). */
snap_status snap_decode_step_noalloc(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                                     const int32_t* n_topk, int32_t n, const int32_t* slot_ids, const void* q,
                                     const void* k_new, const void* v_new, void* out, int32_t out_dtype,
                                     void* stream);

/* The decode position moves on by one token (Sec. III-C: each generated token
 * takes the next position, and the ring row follows from it):
 * pos[slot_ids[b]] += 1 for b < n (once per decode step, after every layer).
 * pos is device int32[n_slots]; slot ids outside [0, n_slots) are skipped. */
snap_status snap_advance(int32_t* pos, int32_t n_slots, int32_t n, const int32_t* slot_ids,
                         void* stream);

/* ---- rotary positions ------------------------------------------------------
 * The compression and attention calls take queries and keys that already carry
 * their positions.  snap_rope puts them there: each pair (x1, x2) of a head's
 * rotated dims turns by the angle position * f_i,
 *   y1 = a (x1 cos - x2 sin),  y2 = a (x2 cos + x1 sin),
 * with f_i = base^(-2i / rot_dim) changed by a rule for contexts longer than
 * the model was trained on. */
typedef enum {
  SNAP_ROPE_HALVES = 0, /* pair i: dims (i, i + rot_dim / 2) of the rotated part */
  SNAP_ROPE_PAIRS = 1   /* pair i: dims (2i, 2i + 1) of the rotated part         */
} snap_rope_layout;

typedef enum {
  SNAP_ROPE_PLAIN = 0,    /* f_i                                                */
  SNAP_ROPE_DIVIDE = 1,   /* f_i / factor: positions divided by factor          */
  SNAP_ROPE_BY_TURNS = 2, /* w f_i + (1 - w) f_i / factor, w from the turns that
                             pair i makes over orig_len positions: 0 up to
                             low_turns, 1 from high_turns, linear between       */
  SNAP_ROPE_BY_INDEX = 3  /* the same, w linear in i: 1 up to lo = max(0,
                             floor(at(high_turns))), 0 from hi = min(rot_dim-1,
                             ceil(at(low_turns))), at(t) the (real) index that
                             makes t turns over orig_len positions              */
} snap_rope_rule;

typedef struct {
  int32_t rot_start;  /* first rotated dim of a head                             */
  int32_t rot_dim;    /* rotated dims: even, 2..128; the others are copied       */
  int32_t layout;     /* snap_rope_layout                                        */
  int32_t rule;       /* snap_rope_rule                                          */
  float base;         /* > 1                                                     */
  float factor;       /* >= 1 (every rule but PLAIN)                             */
  float low_turns;    /* 0 < low_turns < high_turns (BY_TURNS, BY_INDEX)         */
  float high_turns;
  int32_t orig_len;   /* >= 1 (BY_TURNS, BY_INDEX)                               */
  float amplitude;    /* a, > 0 (1: a rotation)                                  */
} snap_rope_params;

/* Heads to rotate: x -> y, [sequence][head][token][d] with any strides (in
 * elements) of the first three; the d dims of a head are contiguous.  y may be
 * x with the same strides (in place: only the rotated dims are touched);
 * otherwise the memory x spans and the memory y spans must be disjoint.
 * Along sizes of more than 1, from the smallest on, each stride of y reaches past
 * all that the smaller ones span (so that no outputs share elements: any slice,
 * permutation or reversal of a tensor).  What is written for one operand must not
 * be read or written for the other. */
typedef struct {
  const void* x;
  void* y;
  int64_t x_stride[3]; /* sequence, head, token */
  int64_t y_stride[3];
  int32_t n_heads;
} snap_rope_heads;

/* Rotates the heads of q and (unless NULL) of k, both of width d and type
 * dtype (SNAP_F32 or SNAP_BF16), in one launch (two where one of them is in
 * place, the other not, and dims are left unrotated).  Token t < lengths[b] (max_len
 * when lengths is NULL; lengths are clamped to [0, max_len]) of sequence b is
 * at position pos[slot_ids[b]] + t, or at t when pos is NULL (slot_ids and
 * n_slots are then not read); tokens past it are neither read nor written, nor
 * are sequences whose slot id is outside [0, n_slots).  Angles are formed in
 * 64 bits and the products in 32; each output is rounded once.  n_seq == 0 is a
 * no-op. */
snap_status snap_rope(const snap_rope_params* r, int32_t dtype, int32_t n_seq, int32_t max_len, int32_t d,
                      const int32_t* pos, int32_t n_slots, const int32_t* slot_ids, const int32_t* lengths,
                      const snap_rope_heads* q, const snap_rope_heads* k, void* stream);

/* ---- paged cache -----------------------------------------------------------
 * A cache of growing length beside the fixed one: layers that are not
 * compressed at the end of prefill, and sequences that are cut back to the
 * budget sink + recent + topk later, by the attention their rows received.
 * Rows live in pages of page_size rows; row r of slot s is row r % page_size of
 * page page_table[s][r / page_size], for every KV head alike.
 *   k      [n_pages][n_kv_heads][page_size][d_qk] kv_dtype
 *   v      [n_pages][n_kv_heads][page_size][d_v]  kv_dtype; NULL when v_in_k
 *   k_scale, v_scale [n_slots][n_kv_heads] fp32: fp8 only, set by the caller
 *   token  [n_pages][n_kv_heads][page_size] int32: the position of the token in
 *          each row (eviction leaves each KV head its own tokens); NULL when
 *          nothing is evicted
 *   weight [n_pages][n_kv_heads][page_size] fp32: the attention the row has
 *          received so far; NULL when it is not kept
 *   page_table [n_slots][max_pages] int32
 * A page id outside [0, n_pages) is a page that is not there: rows in it are
 * not written and receive no attention.  Slots may share pages that none of
 * them writes to, weighs or evicts from.
 * Counters of a slot (device int32[n_slots], caller-owned, shared by every
 * layer): rows[slot] the rows it holds, which is the row of the token being
 * decoded; pos[slot] that token's position.  snap_advance moves each of them on
 * after a step.  The two differ once rows have been evicted.
 * Of snap_params the paged calls take the head layout, widths, types, sm_scale
 * and kv_reuse, and eviction the budget; fp8_qk must be 0. */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int32_t* token;
  float* weight;
  const int32_t* page_table;
  int32_t n_slots;
  int32_t n_pages;
  int32_t page_size; /* a power of two, 16..4096 */
  int32_t max_pages; /* max_pages * page_size <= 2^28 */
} snap_paged_cache;

/* Stores new tokens: token t < lengths[b] (max_len when lengths is NULL) of
 * sequence b goes to row rows[slot] + t of its slot, with token = pos[slot] + t
 * and weight = weight_new[b][g][t] (0 when weight_new is NULL or the value is
 * not finite, as snap_compress's pooled_out is outside the candidates).
 *   k_new [n][n_kv_heads][max_len][d_qk] in_dtype, v_new likewise (NULL when
 *   v_in_k), at strides k_stride / v_stride (host arrays: sequence, head, token
 *   in elements, multiples of 16 bytes along sizes of more than 1; NULL:
 *   contiguous),
 *   weight_new [n][n_kv_heads][max_len] fp32, contiguous.
 * Sequences with rows[slot] < 0 and rows past the page table are skipped.  rows
 * and pos are left as they are; pos may be NULL when the cache has no token
 * array.  The sequences' slots must be distinct. */
snap_status snap_paged_append(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                              const int32_t* pos, int32_t n, const int32_t* slot_ids, const int32_t* lengths,
                              int32_t max_len, const void* k_new, const int64_t* k_stride, const void* v_new,
                              const int64_t* v_stride, const float* weight_new, void* stream);

/* Bytes of workspace snap_paged_decode_attn / _step need for n sequences of at
 * most max_rows rows (the new one included); no fewer than for fewer sequences
 * or rows, nor with weigh than without.  With weigh it holds the logits: n x
 * n_q_heads x max_rows x 4 bytes.  0 on invalid parameters. */
size_t snap_paged_decode_workspace(const snap_params* p, int32_t n, int32_t max_rows, int32_t weigh);

/* Attention of one new token per sequence (already stored) over rows
 * [0, min(rows[slot] + 1, max_rows)) of its slot: out[b][h] =
 * sum_j softmax_j(sm_scale q.k_j) v_j, zero for a sequence without rows.
 * max_rows (host, at most max_pages * page_size) bounds the rows of every
 * sequence of the call; it sizes the launch and the workspace, work follows the
 * rows that are there.  weigh = 1: softmax_j summed over the query heads of each
 * KV head is added to weight of row j (the slots of the call are then distinct).
 *   q   [n][n_q_heads][d_qk] in_dtype, out [n][n_q_heads][d_v] out_dtype,
 *   workspace >= snap_paged_decode_workspace(p, n, max_rows, weigh) bytes,
 *             256-byte aligned; its contents on entry do not matter. */
snap_status snap_paged_decode_attn(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                   int32_t out_dtype, int32_t weigh, void* workspace, size_t ws_bytes, void* stream);

/* snap_paged_append of one token per sequence (k_new [n][n_kv_heads][d_qk],
 * v_new [n][n_kv_heads][d_v], contiguous; weight 0) followed by
 * snap_paged_decode_attn: the same results and cache contents.  The slots of the
 * call are distinct. */
snap_status snap_paged_decode_step(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                                   const int32_t* pos, int32_t n, const int32_t* slot_ids, int32_t max_rows,
                                   const void* q, const void* k_new, const void* v_new, void* out, int32_t out_dtype,
                                   int32_t weigh, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of workspace snap_paged_evict needs; no fewer than for fewer sequences or
 * rows.  0 on invalid parameters. */
size_t snap_paged_evict_workspace(const snap_params* p, int32_t n, int32_t max_rows);

/* Cuts slots back to the budget B = sink + recent + topk, between two steps
 * (rows[slot] rows held, pos[slot] the next position).  A slot of more than B
 * rows keeps, per KV head, the rows with token < sink or token >= pos - recent
 * (the first B of them by row, should there be more) and the heaviest others
 * up to B rows in all (equal weights: the lower row; NaN and negative weights
 * count as 0).  Kept rows below B stay where they are; the j-th kept row from B
 * on moves to the j-th row below B that was not kept, with its token and weight.
 * Rows from B on are left as they were.  A row in a page that is not there is not
 * kept, and none moves into it: where m rows below B are such, B - m are kept.
 *   rows_out [n_slots] int32: min(rows, B) of the call's slots, so that one below
 *            0 stays so (the same from every layer; rows itself is left, so that
 *            every layer sees it),
 *   kept_out optional [n][n_kv_heads][B] int32: the row whose contents are now
 *            in each row, -1 past the rows held and where the page is not there
 *            (NULL to skip),
 *   max_rows (host, at most max_pages * page_size): rows past it are not looked
 *            at: those from B on are not kept, those below B stay where they are,
 *   workspace >= snap_paged_evict_workspace(p, n, max_rows) bytes, 256-byte
 *             aligned; its contents on entry do not matter.
 * The cache needs token and weight; the slots must be distinct and must not
 * share pages; rows_out must not alias rows. */
snap_status snap_paged_evict(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                             const int32_t* pos, int32_t* rows_out, int32_t n, const int32_t* slot_ids,
                             int32_t max_rows, int32_t* kept_out, void* workspace, size_t ws_bytes, void* stream);

/* Stores the tokens of a packed batch by a map (snap_pages_map's): token i < tokens
 * of the batch goes to row row_of[i] (page * page_size + row of the page) of every
 * KV head, with token = pos_of[i] and weight 0.  Its scales (fp8) are those of slot
 * slot_ids[seq_of[i]].
 *   k_new [tokens][n_kv_heads][d_qk] in_dtype, v_new likewise (NULL when v_in_k),
 *   at strides k_stride / v_stride (host arrays: token, head in elements, multiples
 *   of 16 bytes along sizes of more than 1; NULL: contiguous).
 * A token whose row is outside [0, n_pages * page_size), whose sequence is outside
 * [0, n) or whose slot is outside [0, n_slots) is not stored.  The rows must be
 * distinct.  pos_of may be NULL when the cache has no token array. */
snap_status snap_paged_append_mapped(const snap_params* p, const snap_paged_cache* cache, int32_t n,
                                     const int32_t* slot_ids, int32_t tokens, const int32_t* seq_of,
                                     const int32_t* row_of, const int32_t* pos_of, const void* k_new,
                                     const int64_t* k_stride, const void* v_new, const int64_t* v_stride, void* stream);

/* ---- page tables -----------------------------------------------------------
 * The pages of a paged or block cache handed out and taken back on the device, so
 * that a serving step needs no host round trip for them.
 *   page_table [n_slots][max_pages] int32: as in the caches
 *   held       [n_slots] int32: the pages that each slot has, entries [0, held)
 *   free_pages [n_pages] int32: the pages nobody has are entries [0, n_free)
 *   n_free     [1] int32
 * All device memory of the caller, filled once: held 0, page_table -1, free_pages
 * every page, n_free n_pages.  A slot's pages are its own: pages shared between
 * slots are not counted here and must not be handed back. */
typedef struct {
  int32_t* page_table;
  int32_t* held;
  int32_t* free_pages;
  int32_t* n_free;
  int32_t n_slots;
  int32_t n_pages;   /* n_pages * page_size < 2^31 */
  int32_t page_size; /* a power of two, 16..4096 */
  int32_t max_pages; /* max_pages * page_size <= 2^28 */
} snap_page_pool;

/* Room for lengths[b] (len when lengths is NULL) more rows behind the rows[slot]
 * that slot slot_ids[b] holds: the pages it lacks up to then are taken off the end
 * of the free list and entered behind those it has.  Sequences are served in order
 * of b, each whole or not at all: b is served when its pages and those of all
 * sequences before it, served or not, are free together, or when it lacks none;
 * one that wants more than max_pages is not and does not count.
 *   short_out [n] int32: the pages b lacks (0: served), optional.
 * Sequences with a slot id out of range or rows[slot] < 0 are skipped (short 0).
 * A slot named again is served as by a call of its own behind: the sequence lacks what
 * those before it left it to lack.  One workgroup: a call is a few microseconds, 20 where
 * it hands out 48000 pages, and longer where it names a slot twice. */
snap_status snap_pages_reserve(const snap_page_pool* pool, const int32_t* rows, int32_t n, const int32_t* slot_ids,
                               const int32_t* lengths, int32_t len, int32_t* short_out, void* stream);

/* Takes back the pages behind the rows[slot] rows that each slot holds (all of them
 * where that is 0 or less): their entries become -1, and they go to the end of the
 * free list in the order that undoes snap_pages_reserve.  After an eviction, or with
 * rows = 0 at a sequence's end.  (A slot named twice gives them once, where it is named
 * last.) */
snap_status snap_pages_release(const snap_page_pool* pool, const int32_t* rows, int32_t n, const int32_t* slot_ids,
                               void* stream);

/* The map of a packed batch whose sequence b has lengths[b] tokens (negative: none)
 * behind the rows[slot] it holds, from the page table as it is:
 *   starts [n + 1] int32: the batch's first token of each sequence, then their sum
 *          (none above tokens),
 *   seq_of, row_of, pos_of [tokens] int32: each token's sequence b, its physical row
 *          (page * page_size + row of the page; -1 where there is no page) and its
 *          position pos[slot] + t (rows[slot] + t when pos is NULL).
 * Entries past the batch's tokens are -1, -1 and 0.  A sequence with a slot id out
 * of range or rows[slot] < 0 has rows -1 and positions 0.  tokens (host) is the
 * room in the maps; tokens past it are left out.  pool's held and free list are not
 * read and may be NULL here. */
snap_status snap_pages_map(const snap_page_pool* pool, const int32_t* rows, const int32_t* pos, int32_t n,
                           const int32_t* slot_ids, const int32_t* lengths, int32_t tokens, int32_t* starts,
                           int32_t* seq_of, int32_t* row_of, int32_t* pos_of, void* stream);

/* ---- block cache -----------------------------------------------------------
 * A paged cache that only grows, whose rows stand in blocks of `block` tokens: in 8
 * bits with a scale for each block and KV head, formed from the block's own values
 * (nothing to guess, nothing saturates), or in bf16; with bounds of each block's
 * keys, a step may read only the blocks that can matter to its queries.
 *   k, v   [n_pages][n_kv_heads][page_size][d] kv_dtype: SNAP_INT8, SNAP_FP8_E4M3 or
 *          SNAP_BF16 (inputs are bf16; d_qk = d_v = 64 or 128)
 *   k_scale, v_scale [n_pages][n_kv_heads][page_size / block] fp32 (8 bits; NULL: bf16)
 *   k_tail, v_tail   [n_slots][n_kv_heads][block][d] bf16 (8 bits; NULL: bf16): the
 *          rows of the block that the slot's newest token is in, row r at r % block,
 *          as they came.  Until a block is whole it has no codes, and while it is the
 *          newest token's it is attended from here.
 *   bound  [n_pages][n_kv_heads][page_size / block][2][d] int8, and
 *   bound_scale [n_pages][n_kv_heads][page_size / block] fp32: of the whole blocks'
 *          keys, the least (rounded down) and the largest (rounded up) of every dim,
 *          in units of bound_scale; NULL (both) where nothing is selected
 * A whole block's scale is s = amax * fl(1 / 127) (int8, and bounds) or
 * amax * fl(1 / 448) (E4M3), fl and the product in fp32, amax the largest magnitude
 * of its finite values; at least 2^-126, and 1 where amax is 0.  Codes are x / s (fp32
 * quotient) rounded to nearest even, saturating; NaN is the code 0 in int8, E4M3's NaN
 * code there, and no bound.  So codes and scales do not
 * depend on how the tokens were split into calls.
 * Page ids outside [0, n_pages) are pages that are not there: nothing is stored in
 * their rows (nor kept in the tail for them), and they receive no attention.  Slots
 * may share pages of whole blocks that none of them writes to. */
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  void* k_tail;
  void* v_tail;
  void* bound;
  float* bound_scale;
  const int32_t* page_table;
  int32_t n_slots;
  int32_t n_pages;
  int32_t page_size; /* a power of two, block..4096 */
  int32_t max_pages; /* max_pages * page_size <= 2^28 */
  int32_t block;     /* 32, 64 or 128 */
} snap_block_cache;

/* Stores new tokens behind the rows[slot] rows held: token t < lengths[b] (max_len
 * when lengths is NULL) of sequence b in row rows[slot] + t.
 *   starts NULL: k_new [n][n_kv_heads][max_len][d], v_new likewise, at strides
 *     (host arrays: sequence, head, token in elements, multiples of 16 bytes along
 *     sizes of more than 1; NULL: contiguous);
 *   starts [n + 1] (device int32, as snap_pages_map's): a packed batch of `tokens`
 *     tokens, k_new [tokens][n_kv_heads][d]; sequence b has tokens starts[b] ..
 *     starts[b + 1] - 1 (at most max_len of them, a bound that sizes the launch: a
 *     near one spares workgroups; starts outside [0, tokens] are clamped); lengths
 *     is then NULL, and of the strides the sequence's is not read (NULL: contiguous).
 * Sequences with rows[slot] < 0 and rows past the page table are skipped.  rows is
 * left as it is.  The slots must be distinct. */
snap_status snap_block_append(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                              const int32_t* slot_ids, const int32_t* lengths, const int32_t* starts, int32_t tokens,
                              int32_t max_len, const void* k_new, const int64_t* k_stride, const void* v_new,
                              const int64_t* v_stride, void* stream);

/* Blocks that a selection lists at most for a sequence and KV head:
 * ceil(sink / block) + ceil((recent - 1) / block) + ceil(topk / block).  0 on invalid
 * parameters. */
int32_t snap_block_chosen(const snap_params* p, int32_t block);

/* Bytes of workspace snap_block_decode_attn / _step need for n sequences of at most
 * max_rows rows (the new one included); no fewer than for fewer sequences or rows.
 * 0 on invalid parameters. */
size_t snap_block_decode_workspace(const snap_params* p, int32_t n, int32_t max_rows, int32_t block, int32_t select);

/* Attention of one new token per sequence (already stored), at row r = rows[slot],
 * over the rows [0, r] of its slot (select = 0): out[b][h] = sum_j softmax_j(sm_scale
 * q.k_j) v_j, zero for a sequence without rows; blocks before the new token's by
 * their codes, its own by its rows as they came.
 * Values of every size carry the errors of fp32 sums.  Rows whose share of the
 * softmax is below 2^-120 may count as none; an infinite value makes its dim of out
 * infinite, or NaN beside one of the other sign or where its share is below 2^-80.
 * select = 1: over the new token's block and, of the blocks before it,
 *   those with one of the first `sink` rows or of the last `recent` ones, and
 *   the ceil(topk / block) others of the largest score (equal scores: the lower
 *   block),
 * for each KV head.  The score estimates the largest product that a query of the KV
 * head's group may have in a block, formed in whole numbers: with a query's codes a_d =
 * round(q_d / u), u its scale (as a block's in int8), and the block's bounds,
 *   score = bound_scale * max_h u_h * sum_d (a_d > 0 ? a_d largest_d : a_d least_d).
 * It is an upper bound for the rounded query alone: a product q.k may exceed it by half
 * a code's step a dim, u / 2 sum_d |k_d|, by the roundings of fp32 (bounds beyond +-127
 * are clamped), and where keys are infinite (they count as 127 * bound_scale).
 * max_rows (host, at most max_pages * page_size) bounds the rows of every sequence;
 * one that holds more attends those of its whole blocks that lie below max_rows.
 * select needs bounds and at most 32768 blocks (SNAP_ERR_UNSUPPORTED above).
 *   q [n][n_q_heads][d] bf16, out [n][n_q_heads][d] out_dtype,
 *   sel_out [n][n_kv_heads][snap_block_chosen] int32, optional: the blocks selected,
 *           ascending, then -1 (select = 1; not written otherwise),
 *   workspace >= snap_block_decode_workspace(...) bytes, 256-byte aligned; its
 *           contents on entry do not matter. */
snap_status snap_block_decode_attn(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                   int32_t out_dtype, int32_t select, int32_t* sel_out, void* workspace,
                                   size_t ws_bytes, void* stream);

/* snap_block_append of one token per sequence (k_new, v_new [n][n_kv_heads][d],
 * contiguous) followed by snap_block_decode_attn: the same results and cache
 * contents.  The slots of the call are distinct. */
snap_status snap_block_decode_step(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, const void* k_new,
                                   const void* v_new, void* out, int32_t out_dtype, int32_t select, int32_t* sel_out,
                                   void* workspace, size_t ws_bytes, void* stream);

/* Device-side checks of the debug build (libsnapstream_debug.so, built with
 * SNAP_DEBUG_CHECKS): its kernels test the invariants their indexing rests on
 * (keys inside the prompt, kept tokens inside the candidates, rows inside the
 * cache budget, chunk counts within the combine's capacity) and, where one
 * fails, skip the access and record it instead of faulting.  This call waits
 * for the device (hipDeviceSynchronize), stores the recorded bits in *flags (0
 * when none failed) and clears them when reset != 0.  A release build stores
 * 0 and returns SNAP_ERR_UNSUPPORTED.  Bits: 1 score chunk outside the keys,
 * 2 selection past K_eff, 4 kept token outside the candidates, 8 re-scored key
 * outside the candidates, 16 decode rows past the budget, 32 new token's row
 * outside the sink/ring rows, 64 too many split-K chunks, 128 appended row
 * outside the sink/ring rows, 256 prefill block outside the prompt, 512 paged
 * rows cut into more work items than are launched, 1024 evicted rows past their
 * move list, 2048 more blocks selected than a list holds. */
snap_status snap_debug_checks(uint32_t* flags, int32_t reset);

/* Static description of a status code. */
const char* snap_status_str(snap_status s);

/* Message describing the most recent failure on the calling thread ("" if
 * none).  The pointer stays valid until the thread's next library call. */
const char* snap_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SNAPSTREAM_H */
