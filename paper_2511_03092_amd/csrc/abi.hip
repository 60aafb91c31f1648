// abi.hip -- the extern "C" entry points of libsnapstream: host-side argument
// validation, workspace sizing and dispatch to the kernel launchers.  Nothing
// here allocates device memory or synchronises, and every validation runs
// before anything touches the device (the one device query, of
// snap_decode_step_noalloc's scratch address, follows its checks), so every
// validation path can run on a host without a GPU.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include "prefill_order.h"
#include "snap_internal.h"

namespace snap {

static thread_local char g_err[512];

void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
}

static snap_status fail(snap_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Largest second launch-grid dimension (workgroups along y): per-(sequence,
// KV head) and per-(sequence, query head) grids must fit it.
constexpr int kMaxGridY = 65535;
// Sequences of one call of the page-table operators.
constexpr int kMaxSequences = 1 << 20;

// Parameter checks shared by every call.
static snap_status check_params(const snap_params* p) {
  if (!p) return fail(SNAP_ERR_INVALID_ARG, "params is NULL");
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads)
    return fail(SNAP_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)",
                p->n_q_heads, p->n_kv_heads);
  const int G = p->n_q_heads / p->n_kv_heads;
  if (G > 16) return fail(SNAP_ERR_UNSUPPORTED, "at most 16 query heads per KV head (got %d)", G);
  if (p->sink < 0 || p->recent < 1 || p->topk < 0)
    return fail(SNAP_ERR_INVALID_ARG, "need sink >= 0, recent >= 1, topk >= 0 (got %d, %d, %d)", p->sink,
                p->recent, p->topk);
  if ((long long)p->sink + p->recent + p->topk > (1 << 24))
    return fail(SNAP_ERR_INVALID_ARG, "budget sink+recent+topk exceeds 2^24 rows");
  if (p->obs_window < 1) return fail(SNAP_ERR_INVALID_ARG, "obs_window must be >= 1");
  if (p->pool_kernel < 1 || p->pool_kernel > 63 || (p->pool_kernel & 1) == 0)
    return fail(SNAP_ERR_INVALID_ARG, "pool_kernel must be odd in [1, 63] (got %d)", p->pool_kernel);
  if (p->pool != SNAP_POOL_MAX && p->pool != SNAP_POOL_AVG) return fail(SNAP_ERR_INVALID_ARG, "unknown pool type");
  if (p->norm != SNAP_NORM_CAND && p->norm != SNAP_NORM_ROW) return fail(SNAP_ERR_INVALID_ARG, "unknown norm");
  if (!isfinite(p->sm_scale)) return fail(SNAP_ERR_INVALID_ARG, "sm_scale must be finite");
  // a positive scale must keep scale * log2(e) a normal fp32 value: the score
  // kernels form every logit from it and its remainder
  if (p->sm_scale > 0.f && p->sm_scale < 1e-30f)
    return fail(SNAP_ERR_INVALID_ARG, "sm_scale must be <= 0 (the default) or at least 1e-30");
  if (p->fp8_scales != SNAP_FP8_SCALES_GIVEN && p->fp8_scales != SNAP_FP8_SCALES_AMAX)
    return fail(SNAP_ERR_INVALID_ARG, "unknown fp8_scales mode");
  if (p->fp8_qk != 0 && p->fp8_qk != 1) return fail(SNAP_ERR_INVALID_ARG, "fp8_qk must be 0 or 1");
  if (p->kv_reuse != SNAP_KV_AUTO && p->kv_reuse != SNAP_KV_STREAM && p->kv_reuse != SNAP_KV_KEEP)
    return fail(SNAP_ERR_INVALID_ARG, "unknown kv_reuse hint");
  if (p->fp8_qk && !(p->kv_dtype == SNAP_FP8_E4M3 && p->in_dtype == SNAP_BF16 && !p->v_in_k && p->d_qk == 128 &&
                     p->d_v == 128))
    return fail(SNAP_ERR_UNSUPPORTED, "fp8_qk needs bf16 inputs, a GQA fp8 cache and d_qk = d_v = 128");
  const bool dims_ok = (p->d_qk == 64 && p->d_v == 64) || (p->d_qk == 128 && p->d_v == 128) ||
                       (p->d_qk == 576 && p->d_v == 512);
  if (!dims_ok) return fail(SNAP_ERR_UNSUPPORTED, "(d_qk, d_v) must be (64,64), (128,128) or (576,512)");
  if (p->v_in_k != 0 && p->v_in_k != 1) return fail(SNAP_ERR_INVALID_ARG, "v_in_k must be 0 or 1");
  if (p->d_qk == 576 && !p->v_in_k) return fail(SNAP_ERR_UNSUPPORTED, "576/512 is supported as a latent (v_in_k) cache");
  if (p->in_dtype == SNAP_F32) {
    if (p->kv_dtype != SNAP_F32) return fail(SNAP_ERR_UNSUPPORTED, "fp32 inputs need an fp32 cache");
    if (p->d_qk > 128) return fail(SNAP_ERR_UNSUPPORTED, "fp32 inputs support d_qk <= 128");
  } else if (p->in_dtype == SNAP_BF16) {
    if (p->kv_dtype != SNAP_BF16 && p->kv_dtype != SNAP_FP8_E4M3)
      return fail(SNAP_ERR_UNSUPPORTED, "bf16 inputs need a bf16 or fp8 cache");
  } else {
    return fail(SNAP_ERR_INVALID_ARG, "in_dtype must be SNAP_F32 or SNAP_BF16");
  }
  const long rows = (long)G * p->obs_window;
  const long rows_max = p->in_dtype == SNAP_F32 ? 128 : 256;
  if (rows > rows_max)
    return fail(SNAP_ERR_UNSUPPORTED, "G * obs_window = %ld exceeds %ld score rows per KV head", rows, rows_max);
  return SNAP_OK;
}

static snap_status check_cache(const snap_params* p, const snap_cache* c) {
  if (!c) return fail(SNAP_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_slots < 1) return fail(SNAP_ERR_INVALID_ARG, "cache n_slots must be >= 1");
  if (!c->k || !aligned16(c->k)) return fail(SNAP_ERR_INVALID_ARG, "cache k is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!c->v || !aligned16(c->v)))
    return fail(SNAP_ERR_INVALID_ARG, "cache v is NULL or not 16-byte aligned");
  if (p->kv_dtype == SNAP_FP8_E4M3 && (!c->k_scale || (!p->v_in_k && !c->v_scale)))
    return fail(SNAP_ERR_INVALID_ARG, "an fp8 cache needs k_scale and v_scale");
  return SNAP_OK;
}

// One operand of snap_rope: strides that keep distinct outputs apart, and x and
// y either the same or apart.
static snap_status check_rope_heads(const snap_rope_heads* h, const char* name, int32_t n_seq, int32_t max_len, int32_t d,
                                    int elt) {
  if (h->n_heads < 1) return fail(SNAP_ERR_INVALID_ARG, "%s: n_heads must be >= 1", name);
  if (!h->x || !h->y) return fail(SNAP_ERR_INVALID_ARG, "%s: x or y is NULL", name);
  if (((uintptr_t)h->x | (uintptr_t)h->y) & (uintptr_t)(elt - 1))
    return fail(SNAP_ERR_INVALID_ARG, "%s: x or y is not aligned to its elements", name);
  const int64_t size[3] = {n_seq, h->n_heads, max_len};
  // first and last byte (from x, y) that the strides reach; a stride beyond
  // 2^40 elements reaches nothing that exists
  __int128 lo[2] = {0, 0}, hi[2] = {d, d};
  for (int i = 0; i < 3; ++i) {
    const int64_t st[2] = {h->x_stride[i], h->y_stride[i]};
    for (int o = 0; o < 2; ++o) {
      if (size[i] > 1 && (st[o] > ((int64_t)1 << 40) || st[o] < -((int64_t)1 << 40)))
        return fail(SNAP_ERR_INVALID_ARG, "%s: a stride is beyond 2^40 elements", name);
      const __int128 reach = size[i] > 1 ? (__int128)(size[i] - 1) * st[o] : 0;
      (reach < 0 ? lo[o] : hi[o]) += reach;
    }
  }
  // outputs apart: from the smallest stride of y on, each reaches past all that the
  // smaller ones span (any slice, permutation or reversal of a tensor is laid out so)
  __int128 span = d;
  for (unsigned left = (size[0] > 1) | (size[1] > 1) << 1 | (size[2] > 1) << 2; left;) {
    int at = -1;
    for (int i = 0; i < 3; ++i)
      if (left >> i & 1 && (at < 0 || llabs(h->y_stride[i]) < llabs(h->y_stride[at]))) at = i;
    left &= ~(1u << at);
    if (llabs(h->y_stride[at]) < span)
      return fail(SNAP_ERR_INVALID_ARG, "%s: by the strides of y, outputs share elements", name);
    span += (__int128)(size[at] - 1) * llabs(h->y_stride[at]);
  }
  bool same = h->x == h->y;
  for (int i = 0; i < 3; ++i) same = same && (size[i] == 1 || h->x_stride[i] == h->y_stride[i]);
  const __int128 x0 = (__int128)(uintptr_t)h->x + lo[0] * elt, x1 = (__int128)(uintptr_t)h->x + hi[0] * elt;
  const __int128 y0 = (__int128)(uintptr_t)h->y + lo[1] * elt, y1 = (__int128)(uintptr_t)h->y + hi[1] * elt;
  if (!same && x0 < y1 && y0 < x1)
    return fail(SNAP_ERR_INVALID_ARG, "%s: x and y overlap and are not the same", name);
  return SNAP_OK;
}

static snap_status check_paged(const snap_params* p, const snap_paged_cache* c) {
  if (p->fp8_qk) return fail(SNAP_ERR_UNSUPPORTED, "the paged cache has no fp8 query products (fp8_qk)");
  if (!c) return fail(SNAP_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_slots < 1 || c->n_pages < 1 || c->max_pages < 1)
    return fail(SNAP_ERR_INVALID_ARG, "cache n_slots, n_pages and max_pages must be >= 1 (got %d, %d, %d)", c->n_slots,
                c->n_pages, c->max_pages);
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(SNAP_ERR_UNSUPPORTED, "page_size must be a power of two in [16, 4096] (got %d)", c->page_size);
  if ((long long)c->max_pages * c->page_size > (1 << 28))
    return fail(SNAP_ERR_INVALID_ARG, "max_pages * page_size exceeds 2^28 rows");
  if (!c->page_table) return fail(SNAP_ERR_INVALID_ARG, "cache page_table is NULL");
  if (!c->k || !aligned16(c->k)) return fail(SNAP_ERR_INVALID_ARG, "cache k is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!c->v || !aligned16(c->v)))
    return fail(SNAP_ERR_INVALID_ARG, "cache v is NULL or not 16-byte aligned");
  if (!aligned16(c->token) || !aligned16(c->weight))
    return fail(SNAP_ERR_INVALID_ARG, "cache token or weight is not 16-byte aligned");
  if (p->kv_dtype == SNAP_FP8_E4M3 && (!c->k_scale || (!p->v_in_k && !c->v_scale)))
    return fail(SNAP_ERR_INVALID_ARG, "an fp8 cache needs k_scale and v_scale");
  return SNAP_OK;
}

static snap_status check_max_rows(const snap_paged_cache* c, int32_t max_rows) {
  if (max_rows < 1 || (long long)max_rows > (long long)c->max_pages * c->page_size)
    return fail(SNAP_ERR_INVALID_ARG, "max_rows must be in [1, max_pages * page_size = %lld] (got %d)",
                (long long)c->max_pages * c->page_size, max_rows);
  return SNAP_OK;
}

// Checks of snap_paged_decode_attn and, but for the new token, of
// snap_paged_decode_step (n > 0).
static snap_status check_paged_decode(const snap_params* p, const snap_paged_cache* c, const int32_t* rows, int32_t n,
                                      const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                      int32_t out_dtype, int32_t weigh, void* workspace, size_t ws_bytes) {
  snap_status st = check_max_rows(c, max_rows);
  if (st != SNAP_OK) return st;
  if ((long long)n * p->n_q_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_q_heads must be at most %d", kMaxGridY);
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  if (!q || !aligned16(q)) return fail(SNAP_ERR_INVALID_ARG, "q is NULL or not 16-byte aligned");
  if (!out || !aligned16(out)) return fail(SNAP_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
  if (out_dtype != SNAP_F32 && out_dtype != SNAP_BF16) return fail(SNAP_ERR_INVALID_ARG, "out_dtype must be F32 or BF16");
  if (weigh != 0 && weigh != 1) return fail(SNAP_ERR_INVALID_ARG, "weigh must be 0 or 1");
  if (weigh && !c->weight) return fail(SNAP_ERR_INVALID_ARG, "weigh needs the cache's weight array");
  const size_t need = paged_geometry(*p, n, max_rows, weigh != 0).bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  return SNAP_OK;
}

// Checks of the parameters and the cache that the block calls share.
static snap_status check_block(const snap_params* p, const snap_block_cache* c) {
  if (!p) return fail(SNAP_ERR_INVALID_ARG, "params is NULL");
  snap_params as = *p;
  if (as.kv_dtype == SNAP_INT8) as.kv_dtype = SNAP_FP8_E4M3;  // (the other calls have no such cache)
  snap_status st = check_params(&as);
  if (st != SNAP_OK) return st;
  if (p->fp8_qk) return fail(SNAP_ERR_UNSUPPORTED, "the block cache has no fp8 query products (fp8_qk)");
  if (p->in_dtype != SNAP_BF16) return fail(SNAP_ERR_UNSUPPORTED, "the block cache takes bf16 inputs");
  if (p->v_in_k || p->d_qk != p->d_v) return fail(SNAP_ERR_UNSUPPORTED, "the block cache holds 64- or 128-wide keys and values");
  if (!c) return fail(SNAP_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_slots < 1 || c->n_pages < 1 || c->max_pages < 1)
    return fail(SNAP_ERR_INVALID_ARG, "cache n_slots, n_pages and max_pages must be >= 1 (got %d, %d, %d)", c->n_slots,
                c->n_pages, c->max_pages);
  if (c->block != 32 && c->block != 64 && c->block != 128)
    return fail(SNAP_ERR_UNSUPPORTED, "block must be 32, 64 or 128 (got %d)", c->block);
  if (c->page_size < c->block || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(SNAP_ERR_UNSUPPORTED, "page_size must be a power of two in [block, 4096] (got %d)", c->page_size);
  if ((long long)c->max_pages * c->page_size > (1 << 28))
    return fail(SNAP_ERR_INVALID_ARG, "max_pages * page_size exceeds 2^28 rows");
  if ((long long)c->n_pages * (c->page_size / c->block) * p->n_kv_heads > 0x7fffffffll)
    return fail(SNAP_ERR_UNSUPPORTED, "the cache has more than 2^31 - 1 blocks of all KV heads");
  if (!c->page_table) return fail(SNAP_ERR_INVALID_ARG, "cache page_table is NULL");
  if (!c->k || !aligned16(c->k) || !c->v || !aligned16(c->v))
    return fail(SNAP_ERR_INVALID_ARG, "cache k or v is NULL or not 16-byte aligned");
  if (p->kv_dtype != SNAP_BF16) {
    if (!c->k_scale || !c->v_scale) return fail(SNAP_ERR_INVALID_ARG, "an 8-bit cache needs k_scale and v_scale");
    if (!c->k_tail || !aligned16(c->k_tail) || !c->v_tail || !aligned16(c->v_tail))
      return fail(SNAP_ERR_INVALID_ARG, "an 8-bit cache needs k_tail and v_tail, 16-byte aligned");
  }
  if (!c->bound != !c->bound_scale || !aligned16(c->bound))
    return fail(SNAP_ERR_INVALID_ARG, "bound and bound_scale come together, bound 16-byte aligned");
  return SNAP_OK;
}

// Checks of snap_block_decode_attn and, but for the new token, of
// snap_block_decode_step (n > 0).
static snap_status check_block_decode(const snap_params* p, const snap_block_cache* c, const int32_t* rows, int32_t n,
                                      const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                      int32_t out_dtype, int32_t select, void* workspace, size_t ws_bytes) {
  if (max_rows < 1 || (long long)max_rows > (long long)c->max_pages * c->page_size)
    return fail(SNAP_ERR_INVALID_ARG, "max_rows must be in [1, max_pages * page_size = %lld] (got %d)",
                (long long)c->max_pages * c->page_size, max_rows);
  if ((long long)n * p->n_q_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_q_heads must be at most %d", kMaxGridY);
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  if (!q || !aligned16(q)) return fail(SNAP_ERR_INVALID_ARG, "q is NULL or not 16-byte aligned");
  if (!out || !aligned16(out)) return fail(SNAP_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
  if (out_dtype != SNAP_F32 && out_dtype != SNAP_BF16) return fail(SNAP_ERR_INVALID_ARG, "out_dtype must be F32 or BF16");
  if (select != 0 && select != 1) return fail(SNAP_ERR_INVALID_ARG, "select must be 0 or 1");
  if (select && !c->bound) return fail(SNAP_ERR_INVALID_ARG, "select needs the cache's bound and bound_scale");
  if (select && max_rows / c->block > kBlockMost)
    return fail(SNAP_ERR_UNSUPPORTED, "select takes at most %d blocks of a sequence (got %d)", kBlockMost, max_rows / c->block);
  const size_t need = block_geometry(*p, n, max_rows, c->block, select != 0).bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  return SNAP_OK;
}

static snap_status check_pool(const snap_page_pool* c, bool counts) {
  if (!c) return fail(SNAP_ERR_INVALID_ARG, "pool is NULL");
  if (c->n_slots < 1 || c->n_pages < 1 || c->max_pages < 1)
    return fail(SNAP_ERR_INVALID_ARG, "pool n_slots, n_pages and max_pages must be >= 1 (got %d, %d, %d)", c->n_slots,
                c->n_pages, c->max_pages);
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return fail(SNAP_ERR_UNSUPPORTED, "page_size must be a power of two in [16, 4096] (got %d)", c->page_size);
  if ((long long)c->max_pages * c->page_size > (1 << 28))
    return fail(SNAP_ERR_INVALID_ARG, "max_pages * page_size exceeds 2^28 rows");
  if ((long long)c->n_pages * c->page_size > 0x7fffffffll)
    return fail(SNAP_ERR_UNSUPPORTED, "n_pages * page_size must be below 2^31");
  if (!c->page_table) return fail(SNAP_ERR_INVALID_ARG, "pool page_table is NULL");
  if (counts && (!c->held || !c->free_pages || !c->n_free))
    return fail(SNAP_ERR_INVALID_ARG, "pool held, free_pages or n_free is NULL");
  return SNAP_OK;
}

}  // namespace snap

using namespace snap;

extern "C" {

const char* snap_status_str(snap_status s) {
  switch (s) {
    case SNAP_OK: return "ok";
    case SNAP_ERR_INVALID_ARG: return "invalid argument";
    case SNAP_ERR_UNSUPPORTED: return "unsupported configuration";
    case SNAP_ERR_WORKSPACE: return "workspace missing or too small";
    case SNAP_ERR_HIP: return "HIP launch error";
  }
  return "unknown status";
}

const char* snap_last_error(void) { return g_err; }

size_t snap_compress_workspace(const snap_params* p, int32_t n_seq, int32_t max_len) {
  if (check_params(p) != SNAP_OK || n_seq < 0 || max_len < 1) return 0;
  return compress_geometry(*p, n_seq, max_len).compress_bytes;
}

size_t snap_decode_workspace(const snap_params* p, int32_t n) {
  if (check_params(p) != SNAP_OK || n < 0) return 0;
  return decode_geometry(*p, n).decode_bytes;
}

snap_status snap_compress(const snap_params* p, const snap_cache* cache, int32_t* pos, int32_t* n_topk,
                          int32_t n_seq, const int32_t* slot_ids, const int32_t* lengths, int32_t max_len,
                          const void* q_obs, const void* k, const void* v, int32_t* sel_out, float* pooled_out,
                          void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_cache(p, cache)) != SNAP_OK) return st;
  if (n_seq < 0) return fail(SNAP_ERR_INVALID_ARG, "n_seq must be >= 0");
  if (n_seq == 0) return SNAP_OK;
  if (max_len < 1 || max_len > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "max_len must be in [1, 2^28]");
  if ((long long)n_seq * p->n_kv_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n_seq * n_kv_heads must be at most %d", kMaxGridY);
  if (!pos || !n_topk || !slot_ids || !lengths) return fail(SNAP_ERR_INVALID_ARG, "pos/n_topk/slot_ids/lengths NULL");
  if (!q_obs || !aligned16(q_obs)) return fail(SNAP_ERR_INVALID_ARG, "q_obs is NULL or not 16-byte aligned");
  if (!k || !aligned16(k)) return fail(SNAP_ERR_INVALID_ARG, "k is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v || !aligned16(v))) return fail(SNAP_ERR_INVALID_ARG, "v is NULL or not 16-byte aligned");
  if (p->v_in_k && v) return fail(SNAP_ERR_INVALID_ARG, "v must be NULL for a latent (v_in_k) cache");
  if ((sel_out && !aligned16(sel_out)) || (pooled_out && !aligned16(pooled_out)))
    return fail(SNAP_ERR_INVALID_ARG, "sel_out/pooled_out must be 16-byte aligned");
  const size_t need = compress_geometry(*p, n_seq, max_len).compress_bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  st = launch_compress(*p, *cache, pos, n_topk, n_seq, slot_ids, lengths, max_len, q_obs, k, v, sel_out, pooled_out,
                       workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

size_t snap_prefill_workspace(const snap_params* p, int32_t n_seq, int32_t max_len) {
  if (check_params(p) != SNAP_OK || n_seq < 0 || max_len < 1) return 0;
  return prefill_geometry(*p, n_seq, max_len).prefill_bytes;
}

// Checks shared by snap_prefill and snap_prefill_attn.
static snap_status check_prefill(const snap_params* p, int32_t n_seq, const int32_t* lengths, int32_t max_len,
                                 const void* q, const void* k, const void* v, void* out, void* workspace,
                                 size_t ws_bytes) {
  if (p->in_dtype != SNAP_BF16) return fail(SNAP_ERR_UNSUPPORTED, "snap_prefill takes bf16 inputs");
  if (p->v_in_k || p->d_qk != p->d_v || (p->d_qk != 64 && p->d_qk != 128))
    return fail(SNAP_ERR_UNSUPPORTED, "snap_prefill supports d_qk == d_v in {64, 128} with a separate V");
  const int G = p->n_q_heads / p->n_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8 && G != 16)
    return fail(SNAP_ERR_UNSUPPORTED, "snap_prefill supports 1, 2, 4, 8 or 16 query heads per KV head (got %d)", G);
  if (n_seq < 0) return fail(SNAP_ERR_INVALID_ARG, "n_seq must be >= 0");
  if (n_seq == 0) return SNAP_OK;
  if (max_len < 1 || max_len > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "max_len must be in [1, 2^28]");
  const long long groups = (long long)n_seq * p->n_kv_heads;
  if (groups > kMaxGridY || !prefill_grid_fits(groups, G, max_len))
    return fail(SNAP_ERR_UNSUPPORTED, "n_seq * n_kv_heads (%lld) and max_len (%d) exceed the launch grid", groups,
                max_len);
  if (!lengths) return fail(SNAP_ERR_INVALID_ARG, "lengths is NULL");
  if (!q || !aligned16(q) || !k || !aligned16(k) || !v || !aligned16(v))
    return fail(SNAP_ERR_INVALID_ARG, "q, k and v must be non-NULL and 16-byte aligned");
  if (!out || !aligned16(out)) return fail(SNAP_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
  const size_t need = prefill_geometry(*p, n_seq, max_len).prefill_bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  return SNAP_OK;
}

snap_status snap_prefill_attn(const snap_params* p, int32_t n_seq, const int32_t* lengths, int32_t max_len,
                              const void* q, const void* k, const void* v, void* out, void* workspace,
                              size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_prefill(p, n_seq, lengths, max_len, q, k, v, out, workspace, ws_bytes)) != SNAP_OK) return st;
  if (n_seq == 0) return SNAP_OK;
  st = launch_prefill_attn(*p, n_seq, lengths, max_len, q, k, v, out, false, workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_prefill(const snap_params* p, const snap_cache* cache, int32_t* pos, int32_t* n_topk, int32_t n_seq,
                         const int32_t* slot_ids, const int32_t* lengths, int32_t max_len, const void* q, const void* k,
                         const void* v, void* out, int32_t* sel_out, float* pooled_out, void* workspace,
                         size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_cache(p, cache)) != SNAP_OK) return st;
  if ((st = check_prefill(p, n_seq, lengths, max_len, q, k, v, out, workspace, ws_bytes)) != SNAP_OK) return st;
  if (n_seq == 0) return SNAP_OK;
  if (!pos || !n_topk || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "pos/n_topk/slot_ids NULL");
  if ((sel_out && !aligned16(sel_out)) || (pooled_out && !aligned16(pooled_out)))
    return fail(SNAP_ERR_INVALID_ARG, "sel_out/pooled_out must be 16-byte aligned");
  st = launch_prefill(*p, *cache, pos, n_topk, n_seq, slot_ids, lengths, max_len, q, k, v, out, sel_out, pooled_out,
                      workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_cache_append(const snap_params* p, const snap_cache* cache, const int32_t* pos, int32_t n,
                              const int32_t* slot_ids, const void* k_new, const void* v_new, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_cache(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if (!pos || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "pos/slot_ids NULL");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v_new || !aligned16(v_new)))
    return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  st = launch_append(*p, *cache, pos, n, slot_ids, k_new, v_new, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_decode_attn(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                             const int32_t* n_topk, int32_t n, const int32_t* slot_ids, const void* q, void* out,
                             int32_t out_dtype, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_cache(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if ((long long)n * p->n_q_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_q_heads must be at most %d", kMaxGridY);
  if (!pos || !n_topk || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "pos/n_topk/slot_ids NULL");
  if (!q || !aligned16(q)) return fail(SNAP_ERR_INVALID_ARG, "q is NULL or not 16-byte aligned");
  if (!out || !aligned16(out)) return fail(SNAP_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
  if (out_dtype != SNAP_F32 && out_dtype != SNAP_BF16) return fail(SNAP_ERR_INVALID_ARG, "out_dtype must be F32 or BF16");
  const size_t need = decode_geometry(*p, n).decode_bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  st = launch_decode(*p, *cache, pos, n_topk, n, slot_ids, q, nullptr, nullptr, out, out_dtype, workspace,
                     (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

// Checks of snap_decode_step and snap_decode_step_noalloc except the
// workspace.
static snap_status check_decode_step(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                                     const int32_t* n_topk, int32_t n, const int32_t* slot_ids, const void* q,
                                     const void* k_new, const void* v_new, void* out, int32_t out_dtype) {
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_cache(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if ((long long)n * p->n_q_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_q_heads must be at most %d", kMaxGridY);
  if (!pos || !n_topk || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "pos/n_topk/slot_ids NULL");
  if (!q || !aligned16(q)) return fail(SNAP_ERR_INVALID_ARG, "q is NULL or not 16-byte aligned");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v_new || !aligned16(v_new)))
    return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  if (!out || !aligned16(out)) return fail(SNAP_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
  if (out_dtype != SNAP_F32 && out_dtype != SNAP_BF16) return fail(SNAP_ERR_INVALID_ARG, "out_dtype must be F32 or BF16");
  return SNAP_OK;
}

snap_status snap_decode_step(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                             const int32_t* n_topk, int32_t n, const int32_t* slot_ids, const void* q,
                             const void* k_new, const void* v_new, void* out, int32_t out_dtype, void* workspace,
                             size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_decode_step(p, cache, pos, n_topk, n, slot_ids, q, k_new, v_new, out, out_dtype);
  if (st != SNAP_OK || n == 0) return st;
  const size_t need = decode_geometry(*p, n).decode_bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  st = launch_decode(*p, *cache, pos, n_topk, n, slot_ids, q, k_new, p->v_in_k ? nullptr : v_new, out, out_dtype,
                     workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_decode_step_noalloc(const snap_params* p, const snap_cache* cache, const int32_t* pos,
                                     const int32_t* n_topk, int32_t n, const int32_t* slot_ids, const void* q,
                                     const void* k_new, const void* v_new, void* out, int32_t out_dtype,
                                     void* stream) {
  g_err[0] = 0;
  snap_status st = check_decode_step(p, cache, pos, n_topk, n, slot_ids, q, k_new, v_new, out, out_dtype);
  if (st != SNAP_OK || n == 0) return st;
  const size_t need = decode_geometry(*p, n).decode_bytes;
  if (need > (size_t)SNAP_NOALLOC_SCRATCH_BYTES)
    return fail(SNAP_ERR_WORKSPACE, "this call needs %zu bytes of scratch; the library's array holds %zu (split the batch)",
                need, (size_t)SNAP_NOALLOC_SCRATCH_BYTES);
  void* scratch = nullptr;
  if ((st = noalloc_scratch(&scratch)) != SNAP_OK) return st;
  st = launch_decode(*p, *cache, pos, n_topk, n, slot_ids, q, k_new, p->v_in_k ? nullptr : v_new, out, out_dtype,
                     scratch, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_rope(const snap_rope_params* r, int32_t dtype, int32_t n_seq, int32_t max_len, int32_t d,
                      const int32_t* pos, int32_t n_slots, const int32_t* slot_ids, const int32_t* lengths,
                      const snap_rope_heads* q, const snap_rope_heads* k, void* stream) {
  g_err[0] = 0;
  if (!r) return fail(SNAP_ERR_INVALID_ARG, "rope params is NULL");
  if (dtype != SNAP_F32 && dtype != SNAP_BF16) return fail(SNAP_ERR_INVALID_ARG, "dtype must be F32 or BF16");
  if (d < 2 || d > 4096) return fail(SNAP_ERR_INVALID_ARG, "d must be in [2, 4096] (got %d)", d);
  if (r->rot_dim < 2 || r->rot_dim > 2 * kRopeMaxPairs || (r->rot_dim & 1))
    return fail(SNAP_ERR_INVALID_ARG, "rot_dim must be even in [2, %d] (got %d)", 2 * kRopeMaxPairs, r->rot_dim);
  if (r->rot_start < 0 || r->rot_start > d - r->rot_dim)
    return fail(SNAP_ERR_INVALID_ARG, "the rotated dims [%d, +%d) are not within d = %d", r->rot_start, r->rot_dim, d);
  if (r->layout != SNAP_ROPE_HALVES && r->layout != SNAP_ROPE_PAIRS) return fail(SNAP_ERR_INVALID_ARG, "unknown rope layout");
  if (r->rule < SNAP_ROPE_PLAIN || r->rule > SNAP_ROPE_BY_INDEX) return fail(SNAP_ERR_INVALID_ARG, "unknown rope rule");
  if (!isfinite(r->base) || !(r->base > 1.f)) return fail(SNAP_ERR_INVALID_ARG, "rope base must be finite and > 1");
  if (!isfinite(r->amplitude) || !(r->amplitude > 0.f))
    return fail(SNAP_ERR_INVALID_ARG, "rope amplitude must be finite and > 0");
  if (r->rule != SNAP_ROPE_PLAIN && (!isfinite(r->factor) || !(r->factor >= 1.f)))
    return fail(SNAP_ERR_INVALID_ARG, "rope factor must be finite and >= 1");
  if (r->rule == SNAP_ROPE_BY_TURNS || r->rule == SNAP_ROPE_BY_INDEX) {
    if (!isfinite(r->high_turns) || !(r->low_turns > 0.f) || !(r->high_turns > r->low_turns))
      return fail(SNAP_ERR_INVALID_ARG, "need 0 < low_turns < high_turns");
    if (r->orig_len < 1) return fail(SNAP_ERR_INVALID_ARG, "orig_len must be >= 1");
  }
  if (n_seq < 0) return fail(SNAP_ERR_INVALID_ARG, "n_seq must be >= 0");
  if (n_seq == 0) return SNAP_OK;
  if (max_len < 1 || max_len > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "max_len must be in [1, 2^28]");
  if ((long long)n_seq * max_len > (1ll << 31) / d)  // at most a thread per token and dim of a head
    return fail(SNAP_ERR_UNSUPPORTED, "n_seq * max_len * d must be at most 2^31 (split the batch)");
  if (pos && (!slot_ids || n_slots < 1)) return fail(SNAP_ERR_INVALID_ARG, "pos needs slot_ids and n_slots >= 1");
  if (!q) return fail(SNAP_ERR_INVALID_ARG, "q is NULL");
  const int elt = dtype == SNAP_F32 ? 4 : 2;
  snap_status st = check_rope_heads(q, "q", n_seq, max_len, d, elt);
  if (st != SNAP_OK) return st;
  if (k && (st = check_rope_heads(k, "k", n_seq, max_len, d, elt)) != SNAP_OK) return st;
  if ((long long)q->n_heads + (k ? k->n_heads : 0) > (1 << 20))
    return fail(SNAP_ERR_UNSUPPORTED, "at most 2^20 heads");
  st = launch_rope(*r, dtype, n_seq, max_len, d, pos, n_slots, slot_ids, lengths, q, k, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_paged_append(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                              const int32_t* pos, int32_t n, const int32_t* slot_ids, const int32_t* lengths,
                              int32_t max_len, const void* k_new, const int64_t* k_stride, const void* v_new,
                              const int64_t* v_stride, const float* weight_new, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_paged(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if (max_len < 1 || max_len > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "max_len must be in [1, 2^28]");
  if ((long long)n * p->n_kv_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_kv_heads must be at most %d", kMaxGridY);
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  if (cache->token && !pos) return fail(SNAP_ERR_INVALID_ARG, "a cache with a token array needs pos");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v_new || !aligned16(v_new)))
    return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  const int per16 = p->in_dtype == SNAP_F32 ? 4 : 8;
  const int32_t size[3] = {n, p->n_kv_heads, max_len};
  for (int i = 0; i < 3; ++i)  // (a stride along a size of 1 says nothing)
    if (size[i] > 1 && ((k_stride && k_stride[i] % per16) || (!p->v_in_k && v_stride && v_stride[i] % per16)))
      return fail(SNAP_ERR_INVALID_ARG, "strides of k_new / v_new must be multiples of 16 bytes");
  st = launch_paged_append(*p, *cache, rows, pos, n, slot_ids, lengths, max_len, k_new, k_stride, v_new, v_stride,
                           weight_new, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

size_t snap_paged_decode_workspace(const snap_params* p, int32_t n, int32_t max_rows, int32_t weigh) {
  if (check_params(p) != SNAP_OK || n < 0 || max_rows < 1 || max_rows > (1 << 28)) return 0;
  if ((long long)n * p->n_q_heads > kMaxGridY) return 0;
  return paged_geometry(*p, n, max_rows, weigh != 0).bytes;
}

snap_status snap_paged_decode_attn(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                   int32_t out_dtype, int32_t weigh, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_paged(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  st = check_paged_decode(p, cache, rows, n, slot_ids, max_rows, q, out, out_dtype, weigh, workspace, ws_bytes);
  if (st != SNAP_OK) return st;
  st = launch_paged_decode(*p, *cache, rows, nullptr, n, slot_ids, max_rows, q, nullptr, nullptr, out, out_dtype,
                           weigh != 0, workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_paged_decode_step(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                                   const int32_t* pos, int32_t n, const int32_t* slot_ids, int32_t max_rows,
                                   const void* q, const void* k_new, const void* v_new, void* out, int32_t out_dtype,
                                   int32_t weigh, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_paged(p, cache)) != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  st = check_paged_decode(p, cache, rows, n, slot_ids, max_rows, q, out, out_dtype, weigh, workspace, ws_bytes);
  if (st != SNAP_OK) return st;
  if (cache->token && !pos) return fail(SNAP_ERR_INVALID_ARG, "a cache with a token array needs pos");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v_new || !aligned16(v_new)))
    return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  st = launch_paged_decode(*p, *cache, rows, pos, n, slot_ids, max_rows, q, k_new, v_new, out, out_dtype, weigh != 0,
                           workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

size_t snap_paged_evict_workspace(const snap_params* p, int32_t n, int32_t max_rows) {
  if (check_params(p) != SNAP_OK || n < 0 || max_rows < 1 || max_rows > (1 << 28)) return 0;
  if ((long long)n * p->n_kv_heads > kMaxGridY) return 0;
  return evict_geometry(*p, n, max_rows).bytes;
}

snap_status snap_paged_evict(const snap_params* p, const snap_paged_cache* cache, const int32_t* rows,
                             const int32_t* pos, int32_t* rows_out, int32_t n, const int32_t* slot_ids,
                             int32_t max_rows, int32_t* kept_out, void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_paged(p, cache)) != SNAP_OK) return st;
  if (!cache->token || !cache->weight) return fail(SNAP_ERR_INVALID_ARG, "eviction needs the cache's token and weight arrays");
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if ((st = check_max_rows(cache, max_rows)) != SNAP_OK) return st;
  if ((long long)n * p->n_kv_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_kv_heads must be at most %d", kMaxGridY);
  if (!rows || !pos || !rows_out || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/pos/rows_out/slot_ids NULL");
  if (rows_out == rows) return fail(SNAP_ERR_INVALID_ARG, "rows_out must not alias rows");
  const size_t need = evict_geometry(*p, n, max_rows).bytes;
  if (!workspace || ((uintptr_t)workspace & 255u) || ws_bytes < need)
    return fail(SNAP_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu)", need, ws_bytes);
  st = launch_paged_evict(*p, *cache, rows, pos, rows_out, n, slot_ids, max_rows, kept_out, workspace,
                          (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_paged_append_mapped(const snap_params* p, const snap_paged_cache* cache, int32_t n,
                                     const int32_t* slot_ids, int32_t tokens, const int32_t* seq_of,
                                     const int32_t* row_of, const int32_t* pos_of, const void* k_new,
                                     const int64_t* k_stride, const void* v_new, const int64_t* v_stride,
                                     void* stream) {
  g_err[0] = 0;
  snap_status st = check_params(p);
  if (st != SNAP_OK) return st;
  if ((st = check_paged(p, cache)) != SNAP_OK) return st;
  if (n < 0 || tokens < 0) return fail(SNAP_ERR_INVALID_ARG, "n and tokens must be >= 0");
  if (n == 0 || tokens == 0) return SNAP_OK;
  if (tokens > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "tokens must be at most 2^28");
  if (p->n_kv_heads > kMaxGridY) return fail(SNAP_ERR_UNSUPPORTED, "n_kv_heads must be at most %d", kMaxGridY);
  if ((long long)cache->n_pages * cache->page_size > 0x7fffffffll)
    return fail(SNAP_ERR_UNSUPPORTED, "n_pages * page_size must be below 2^31");
  if (!slot_ids || !seq_of || !row_of) return fail(SNAP_ERR_INVALID_ARG, "slot_ids/seq_of/row_of NULL");
  if (cache->token && !pos_of) return fail(SNAP_ERR_INVALID_ARG, "a cache with a token array needs pos_of");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!p->v_in_k && (!v_new || !aligned16(v_new)))
    return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  const int per16 = p->in_dtype == SNAP_F32 ? 4 : 8;
  const int32_t size[2] = {tokens, p->n_kv_heads};
  for (int i = 0; i < 2; ++i)
    if (size[i] > 1 && ((k_stride && k_stride[i] % per16) || (!p->v_in_k && v_stride && v_stride[i] % per16)))
      return fail(SNAP_ERR_INVALID_ARG, "strides of k_new / v_new must be multiples of 16 bytes");
  st = launch_paged_append_mapped(*p, *cache, n, slot_ids, tokens, seq_of, row_of, pos_of, k_new, k_stride, v_new,
                                  v_stride, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_pages_reserve(const snap_page_pool* pool, const int32_t* rows, int32_t n, const int32_t* slot_ids,
                               const int32_t* lengths, int32_t len, int32_t* short_out, void* stream) {
  g_err[0] = 0;
  snap_status st = check_pool(pool, true);
  if (st != SNAP_OK) return st;
  if (n < 0 || n > kMaxSequences) return fail(SNAP_ERR_INVALID_ARG, "n must be in [0, %d]", kMaxSequences);
  if (!lengths && len < 0) return fail(SNAP_ERR_INVALID_ARG, "len must be >= 0");
  if (n == 0) return SNAP_OK;
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  st = launch_pages_reserve(*pool, rows, n, slot_ids, lengths, len, short_out, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_pages_release(const snap_page_pool* pool, const int32_t* rows, int32_t n, const int32_t* slot_ids,
                               void* stream) {
  g_err[0] = 0;
  snap_status st = check_pool(pool, true);
  if (st != SNAP_OK) return st;
  if (n < 0 || n > kMaxSequences) return fail(SNAP_ERR_INVALID_ARG, "n must be in [0, %d]", kMaxSequences);
  if (n == 0) return SNAP_OK;
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  st = launch_pages_release(*pool, rows, n, slot_ids, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_pages_map(const snap_page_pool* pool, const int32_t* rows, const int32_t* pos, int32_t n,
                           const int32_t* slot_ids, const int32_t* lengths, int32_t tokens, int32_t* starts,
                           int32_t* seq_of, int32_t* row_of, int32_t* pos_of, void* stream) {
  g_err[0] = 0;
  snap_status st = check_pool(pool, false);
  if (st != SNAP_OK) return st;
  if (n < 0 || n > kMaxSequences) return fail(SNAP_ERR_INVALID_ARG, "n must be in [0, %d]", kMaxSequences);
  if (tokens < 0 || tokens > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "tokens must be in [0, 2^28]");
  if (n > 0 && (!rows || !slot_ids || !lengths)) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids/lengths NULL");
  if (!starts || (tokens > 0 && (!seq_of || !row_of || !pos_of)))
    return fail(SNAP_ERR_INVALID_ARG, "starts/seq_of/row_of/pos_of NULL");
  st = launch_pages_map(*pool, rows, pos, n, slot_ids, lengths, tokens, starts, seq_of, row_of, pos_of,
                        (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_block_append(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                              const int32_t* slot_ids, const int32_t* lengths, const int32_t* starts, int32_t tokens,
                              int32_t max_len, const void* k_new, const int64_t* k_stride, const void* v_new,
                              const int64_t* v_stride, void* stream) {
  g_err[0] = 0;
  snap_status st = check_block(p, cache);
  if (st != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  if (max_len < 1 || max_len > (1 << 28)) return fail(SNAP_ERR_INVALID_ARG, "max_len must be in [1, 2^28]");
  if ((long long)n * p->n_kv_heads > kMaxGridY)
    return fail(SNAP_ERR_UNSUPPORTED, "n * n_kv_heads must be at most %d", kMaxGridY);
  if (!rows || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "rows/slot_ids NULL");
  if (starts && lengths) return fail(SNAP_ERR_INVALID_ARG, "a packed batch (starts) takes no lengths");
  if (starts && tokens < 0) return fail(SNAP_ERR_INVALID_ARG, "tokens must be >= 0");
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!v_new || !aligned16(v_new)) return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  const int32_t size[3] = {starts ? 1 : n, p->n_kv_heads, starts ? tokens : max_len};
  for (int i = 0; i < 3; ++i)
    if (size[i] > 1 && ((k_stride && k_stride[i] % 8) || (v_stride && v_stride[i] % 8)))
      return fail(SNAP_ERR_INVALID_ARG, "strides of k_new / v_new must be multiples of 16 bytes");
  st = launch_block_append(*p, *cache, rows, n, slot_ids, lengths, starts, tokens, max_len, k_new, k_stride, v_new,
                           v_stride, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

int32_t snap_block_chosen(const snap_params* p, int32_t block) {
  if (!p || (block != 32 && block != 64 && block != 128)) return 0;
  if (p->sink < 0 || p->recent < 1 || p->topk < 0 || (long long)p->sink + p->recent + p->topk > (1 << 24)) return 0;
  return block_chosen(*p, block);
}

size_t snap_block_decode_workspace(const snap_params* p, int32_t n, int32_t max_rows, int32_t block, int32_t select) {
  if (!p || n < 0 || max_rows < 1 || max_rows > (1 << 28) || (block != 32 && block != 64 && block != 128)) return 0;
  snap_params as = *p;
  if (as.kv_dtype == SNAP_INT8) as.kv_dtype = SNAP_FP8_E4M3;
  if (check_params(&as) != SNAP_OK || p->d_qk != p->d_v) return 0;
  if ((long long)n * p->n_q_heads > kMaxGridY) return 0;
  return block_geometry(*p, n, max_rows, block, select != 0).bytes;
}

snap_status snap_block_decode_attn(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, void* out,
                                   int32_t out_dtype, int32_t select, int32_t* sel_out, void* workspace,
                                   size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_block(p, cache);
  if (st != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  st = check_block_decode(p, cache, rows, n, slot_ids, max_rows, q, out, out_dtype, select, workspace, ws_bytes);
  if (st != SNAP_OK) return st;
  st = launch_block_decode(*p, *cache, rows, n, slot_ids, max_rows, q, nullptr, nullptr, out, out_dtype, select != 0,
                           sel_out, workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_block_decode_step(const snap_params* p, const snap_block_cache* cache, const int32_t* rows, int32_t n,
                                   const int32_t* slot_ids, int32_t max_rows, const void* q, const void* k_new,
                                   const void* v_new, void* out, int32_t out_dtype, int32_t select, int32_t* sel_out,
                                   void* workspace, size_t ws_bytes, void* stream) {
  g_err[0] = 0;
  snap_status st = check_block(p, cache);
  if (st != SNAP_OK) return st;
  if (n < 0) return fail(SNAP_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return SNAP_OK;
  st = check_block_decode(p, cache, rows, n, slot_ids, max_rows, q, out, out_dtype, select, workspace, ws_bytes);
  if (st != SNAP_OK) return st;
  if (!k_new || !aligned16(k_new)) return fail(SNAP_ERR_INVALID_ARG, "k_new is NULL or not 16-byte aligned");
  if (!v_new || !aligned16(v_new)) return fail(SNAP_ERR_INVALID_ARG, "v_new is NULL or not 16-byte aligned");
  st = launch_block_decode(*p, *cache, rows, n, slot_ids, max_rows, q, k_new, v_new, out, out_dtype, select != 0,
                           sel_out, workspace, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

snap_status snap_debug_checks(uint32_t* flags, int32_t reset) {
  g_err[0] = 0;
  if (!flags) return fail(SNAP_ERR_INVALID_ARG, "flags is NULL");
  *flags = 0;
#ifdef SNAP_DEBUG_CHECKS
  if (hipDeviceSynchronize() != hipSuccess) return fail(SNAP_ERR_HIP, "hipDeviceSynchronize failed");
  const uint32_t c = debug_flags_compress(reset != 0), d = debug_flags_decode(reset != 0),
                 f = debug_flags_prefill(reset != 0), g = debug_flags_paged(reset != 0),
                 e = debug_flags_evict(reset != 0), h = debug_flags_blocks(reset != 0);
  if (c == 0xffffffffu || d == 0xffffffffu || f == 0xffffffffu || g == 0xffffffffu || e == 0xffffffffu ||
      h == 0xffffffffu)
    return fail(SNAP_ERR_HIP, "reading the check words failed");
  *flags = c | d | f | g | e | h;
  return SNAP_OK;
#else
  (void)reset;
  return fail(SNAP_ERR_UNSUPPORTED, "a release build: no device-side checks (build with --debug)");
#endif
}

snap_status snap_advance(int32_t* pos, int32_t n_slots, int32_t n, const int32_t* slot_ids, void* stream) {
  g_err[0] = 0;
  if (n < 0 || n_slots < 1) return fail(SNAP_ERR_INVALID_ARG, "need n >= 0 and n_slots >= 1");
  if (n == 0) return SNAP_OK;
  if (!pos || !slot_ids) return fail(SNAP_ERR_INVALID_ARG, "pos/slot_ids NULL");
  snap_status st = launch_advance(pos, n_slots, n, slot_ids, (hipStream_t)stream);
  if (st == SNAP_ERR_HIP) set_error("kernel launch failed: %s", hipGetErrorString(hipGetLastError()));
  return st;
}

}  // extern "C"
