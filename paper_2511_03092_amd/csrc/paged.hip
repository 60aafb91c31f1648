// paged.hip -- the paged cache: storing new tokens, and attention of one new
// token per sequence over every row its slot holds.
//
//   paged_append   stores the tokens of a prompt or of a step
//   paged_decode   one wave per (work item, query head): online softmax over
//                  the item's rows
//   paged_join     merges the items of a (sequence, query head) -> out
//   paged_weigh    adds the rows' softmax weights to their accumulated ones
//
// Work items.  Sequences are of unequal length and their lengths are on the
// device, so the rows are cut there: every unit (sequence, KV head) takes
// ceil(blocks / C) items of nearly equal length, C the 32-row blocks of all
// units over the items wanted, so that an item is as long as another whatever
// sequence it is of.  Every wave finds its item from the lengths alone.
#include <math.h>

#include "snap_internal.h"

namespace snap {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kBlockRows = 32;  // rows of a block
constexpr int kItemTarget = 2048;

struct PagedArgs {
  const void* q;  // [n][Hq][dk]
  const void* ck;
  const void* cv;
  const float* k_scale;
  const float* v_scale;
  const int32_t* rows;
  const int32_t* slot_ids;
  const int32_t* table;
  float* part;   // [items][G][dv]
  float2* ml;    // [items][G]  (max in log2 units, sum)
  float* z;      // logits in log2 units, [unit][G][its rows, whole blocks]; NULL without weights
  float* weight;
  void* out;
  int n, Hq, Hkv, G, dk, dv, n_slots, n_pages, page_shift, max_pages, max_rows, target, max_items, out_bf16, q_f32;
  float scale;
};

// The rows sequence b attends (0 for a slot id out of range).
__device__ __forceinline__ int rows_of(const PagedArgs& a, int b, int& slot) {
  slot = a.slot_ids[b];
  if (slot < 0 || slot >= a.n_slots) return 0;
  const int r = a.rows[slot];
  return r < 0 ? 0 : (r >= a.max_rows ? a.max_rows : r + 1);
}

__device__ __forceinline__ int wave_sum_i(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
// inclusive prefix sum over the wave
__device__ __forceinline__ int wave_scan_i(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// One sequence of the cut: its blocks, items per unit, the items of the
// sequences before it and the blocks of theirs.
struct PagedSeq {
  int b, slot, len, blocks, items;
  int item0;       // items before the sequence's first
  int64_t block0;  // blocks of the units before its first
};

// Called by a whole wave.  by_item: the sequence that holds item `key`;
// otherwise sequence `key`.  false: there is none.
__device__ __forceinline__ bool paged_seq(const PagedArgs& a, int key, bool by_item, PagedSeq& s) {
  const int lane = tid() & 63;
  int64_t total = 0;
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    int slot;
    const int b = b0 + lane;
    const int nb = b < a.n ? (rows_of(a, b, slot) + kBlockRows - 1) / kBlockRows : 0;
    total += wave_sum_i(nb);
  }
  const int64_t c64 = (total * a.Hkv + a.target - 1) / a.target;
  const int C = c64 < 1 ? 1 : (int)c64;  // blocks an item
  int items_before = 0;
  int64_t blocks_before = 0;
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    int slot = -1;
    const int b = b0 + lane;
    const int len = b < a.n ? rows_of(a, b, slot) : 0;
    const int nb = (len + kBlockRows - 1) / kBlockRows;
    const int ni = (nb + C - 1) / C;
    const int si = wave_scan_i(ni, lane), sb = wave_scan_i(nb, lane);
    const int first = items_before + a.Hkv * (si - ni);
    const bool here = b < a.n && (by_item ? key >= first && key < first + a.Hkv * ni : key == b);
    const uint64_t m = __builtin_amdgcn_ballot_w64(here);
    if (m) {
      const int at = __builtin_ctzll(m);
      s.b = b0 + at;
      s.slot = uniform(__shfl(slot, at));
      s.len = uniform(__shfl(len, at));
      s.blocks = uniform(__shfl(nb, at));
      s.items = uniform(__shfl(ni, at));
      s.item0 = uniform(__shfl(first, at));
      s.block0 = blocks_before + (int64_t)a.Hkv * uniform(__shfl(sb - nb, at));
      return true;
    }
    items_before += a.Hkv * uniform(__shfl(si, 63));
    blocks_before += (int64_t)a.Hkv * uniform(__shfl(sb, 63));
  }
  return false;
}

// Index of row r of (slot, KV head g) among the rows of all pages, or -1 when
// its page is not there.
__device__ __forceinline__ int64_t paged_row(const PagedArgs& a, int slot, int g, int r) {
  const int page = a.table[(size_t)slot * a.max_pages + (r >> a.page_shift)];
  if (page < 0 || page >= a.n_pages) return -1;
  return (((int64_t)page * a.Hkv + g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
}

template <typename KV>
__device__ __forceinline__ float kv_f32(KV x) {
  if constexpr (sizeof(KV) == 4)
    return x;
  else if constexpr (sizeof(KV) == 2)
    return bf16_bits_to_f32(x);
  else
    return e4m3_to_f32(x);
}

template <typename KV>
__global__ __launch_bounds__(64) void paged_decode(PagedArgs a) {
  const int lane = tid(), item = bid_x(), h = bid_y();
  PagedSeq s;
  if (!paged_seq(a, item, true, s)) return;
  if (!debug_check(item < a.max_items, kDbgPagedItem)) return;
  const int local = item - s.item0, g = local / s.items, chunk = local % s.items;
  const int r0 = (int)((int64_t)chunk * s.blocks / s.items) * kBlockRows;
  const int r1 = min(s.len, (int)((int64_t)(chunk + 1) * s.blocks / s.items) * kBlockRows);
  constexpr int kMaxPer = 9;  // dims a lane: 576 / 64
  const int nk = a.dk / 64, nv = a.dv / 64;
  const size_t qo = ((size_t)s.b * a.Hq + g * a.G + h) * a.dk;
  const float ksc = sizeof(KV) == 1 ? a.k_scale[(size_t)s.slot * a.Hkv + g] : 1.f;
  const float vsc = sizeof(KV) == 1 ? (a.cv ? a.v_scale : a.k_scale)[(size_t)s.slot * a.Hkv + g] : 1.f;
  const float xs = a.scale * kLog2e * ksc;
  float q[kMaxPer], acc[kMaxPer];
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i) {
    q[i] = 0.f;
    acc[i] = 0.f;
    if (i < nk)
      q[i] = a.q_f32 ? ((const float*)a.q)[qo + i * 64 + lane] : bf16_bits_to_f32(((const uint16_t*)a.q)[qo + i * 64 + lane]);
  }
  float m = -INFINITY, l = 0.f;
  float* z = a.z ? a.z + ((s.block0 + (int64_t)g * s.blocks) * a.G + (int64_t)h * s.blocks) * kBlockRows : nullptr;
  for (int r = r0; r < r1; ++r) {
    const int64_t row = paged_row(a, s.slot, g, r);
    float x = -INFINITY;
    if (row >= 0) {
      const KV* kp = (const KV*)a.ck + row * a.dk;
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < kMaxPer; ++i)
        if (i < nk) dot = fmaf(q[i], kv_f32<KV>(kp[i * 64 + lane]), dot);
      x = warp_sum(dot) * xs;
      const float mn = fmaxf(m, x);
      if (mn != -INFINITY) {
        const float al = fast_exp2(m - mn), p = fast_exp2(x - mn);
        l = fmaf(l, al, p);
        const KV* vp = a.cv ? (const KV*)a.cv + row * a.dv : kp;
#pragma unroll
        for (int i = 0; i < kMaxPer; ++i)
          if (i < nv) acc[i] = fmaf(acc[i], al, p * kv_f32<KV>(vp[i * 64 + lane]));
        m = mn;
      }
    }
    if (z && lane == 0) z[r] = x;
  }
  const size_t pi = (size_t)item * a.G + h;
  if (lane == 0) a.ml[pi] = make_float2(m, l);
#pragma unroll
  for (int i = 0; i < kMaxPer; ++i)
    if (i < nv) a.part[pi * a.dv + i * 64 + lane] = acc[i] * vsc;
}

// ---------------------------------------------------------------- join
// The largest reference and the sum of a unit's items, for query head h of it.
__device__ __forceinline__ float2 joined_ml(const PagedArgs& a, const PagedSeq& s, int g, int h) {
  const int i0 = s.item0 + g * s.items, lane = tid() & 63;
  float m = -INFINITY;
  for (int i = lane; i < s.items; i += 64) m = fmaxf(m, a.ml[(size_t)(i0 + i) * a.G + h].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.f;
  for (int i = lane; i < s.items; i += 64) {
    const float2 v = a.ml[(size_t)(i0 + i) * a.G + h];
    if (v.x != -INFINITY) l = fmaf(fast_exp2(v.x - m), v.y, l);
  }
  return make_float2(m, warp_sum(l));
}

__global__ __launch_bounds__(64) void paged_join(PagedArgs a) {
  const int lane = tid(), b = bid_x() / a.Hq, qh = bid_x() % a.Hq, g = qh / a.G, h = qh % a.G;
  PagedSeq s;
  if (!paged_seq(a, b, false, s)) return;
  if (s.slot < 0 || s.slot >= a.n_slots) return;
  const float2 ml = joined_ml(a, s, g, h);
  const float inv = ml.y > 0.f ? 1.f / ml.y : 0.f;
  for (int d = lane; d < a.dv; d += 64) {
    float o = 0.f;
    for (int i = 0; i < s.items; ++i) {
      const size_t pi = (size_t)(s.item0 + g * s.items + i) * a.G + h;
      const float mi = a.ml[pi].x;
      if (mi != -INFINITY) o = fmaf(fast_exp2(mi - ml.x), a.part[pi * a.dv + d], o);
    }
    o *= inv;
    const size_t oi = ((size_t)b * a.Hq + qh) * a.dv + d;
    if (a.out_bf16)
      ((uint16_t*)a.out)[oi] = (uint16_t)f32_to_bf16_bits(o);
    else
      ((float*)a.out)[oi] = o;
  }
}

// One thread per row; block x: 256 rows, y: unit.
__global__ __launch_bounds__(256) void paged_weigh(PagedArgs a) {
  const int b = bid_y() / a.Hkv, g = bid_y() % a.Hkv, r = bid_x() * 256 + tid();
  PagedSeq s;
  if (!paged_seq(a, b, false, s)) return;
  const int64_t row = r < s.len ? paged_row(a, s.slot, g, r) : -1;
  const float* z = a.z + (s.block0 + (int64_t)g * s.blocks) * a.G * kBlockRows;
  float w = 0.f;
  for (int h = 0; h < a.G; ++h) {
    const float2 ml = joined_ml(a, s, g, h);
    if (row >= 0 && ml.y > 0.f) w = fmaf(fast_exp2(z[(int64_t)h * s.blocks * kBlockRows + r] - ml.x), 1.f / ml.y, w);
  }
  if (row >= 0) a.weight[row] += w;
}

// ---------------------------------------------------------------- append
struct PagedAppendArgs {
  const void* k_new;
  const void* v_new;
  const float* weight_new;
  void* ck;
  void* cv;
  const float* k_scale;
  const float* v_scale;
  int32_t* token;
  float* weight;
  const int32_t* rows;
  const int32_t* pos;
  const int32_t* slot_ids;
  const int32_t* lengths;
  const int32_t* table;
  int64_t ks[3], vs[3];
  int Hkv, dk, dv, n_slots, n_pages, page_shift, max_pages, max_len;
};

// 8 elements of an input row -> the cache's form (fp8: the codes of x / scale)
template <typename In, typename Out>
__device__ __forceinline__ void store8(const In* src, Out* dst, float scale) {
  if constexpr (sizeof(Out) == 1) {
    const u32x4 raw = *(const u32x4*)src;
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_bits_to_f32(raw[i] & 0xffffu) / scale;
      f[2 * i + 1] = bf16_bits_to_f32(raw[i] >> 16) / scale;
    }
    const u32x2 o = {e4m3x4_hw(f[0], f[1], f[2], f[3]), e4m3x4_hw(f[4], f[5], f[6], f[7])};
    *(u32x2*)dst = o;
  } else {
    *(u32x4*)dst = *(const u32x4*)src;
    if constexpr (sizeof(In) == 4) *(u32x4*)(dst + 4) = *(const u32x4*)(src + 4);
  }
}

// block x: tokens 32x .. 32x + 31, y: KV head, z: sequence
constexpr int kAppendTokens = 32;
template <typename In, typename Out>
__global__ __launch_bounds__(256) void paged_append(PagedAppendArgs a) {
  const int g = bid_y(), b = __builtin_amdgcn_workgroup_id_z();
  const int slot = a.slot_ids[b];
  if (slot < 0 || slot >= a.n_slots) return;
  const int row0 = a.rows[slot];
  if (row0 < 0) return;
  int len = a.lengths ? a.lengths[b] : a.max_len;
  len = len > a.max_len ? a.max_len : len;
  const int64_t room = ((int64_t)a.max_pages << a.page_shift) - row0;
  if (len > room) len = room < 0 ? 0 : (int)room;
  const int kc = a.dk / 8, vc = a.v_new ? a.dv / 8 : 0;
  const float ksc = sizeof(Out) == 1 ? a.k_scale[(size_t)slot * a.Hkv + g] : 1.f;
  const float vsc = sizeof(Out) == 1 && vc ? a.v_scale[(size_t)slot * a.Hkv + g] : 1.f;
  const int t0 = bid_x() * kAppendTokens;
  for (int i = tid(); i < kAppendTokens * (kc + vc); i += 256) {
    const int t = t0 + i / (kc + vc), c = i % (kc + vc);
    if (t >= len) break;
    const int r = row0 + t, page = a.table[(size_t)slot * a.max_pages + (r >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) continue;
    const int64_t row = (((int64_t)page * a.Hkv + g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
    if (c < kc)
      store8<In, Out>((const In*)a.k_new + b * a.ks[0] + g * a.ks[1] + t * a.ks[2] + 8 * c,
                      (Out*)a.ck + row * a.dk + 8 * c, ksc);
    else
      store8<In, Out>((const In*)a.v_new + b * a.vs[0] + g * a.vs[1] + t * a.vs[2] + 8 * (c - kc),
                      (Out*)a.cv + row * a.dv + 8 * (c - kc), vsc);
    if (c == 0) {
      if (a.token) a.token[row] = a.pos[slot] + t;
      if (a.weight) {
        // not finite: by its bits, the build lets float compares assume no NaN
        float w = a.weight_new ? a.weight_new[((size_t)b * a.Hkv + g) * a.max_len + t] : 0.f;
        if ((__float_as_uint(w) & 0x7f800000u) == 0x7f800000u) w = 0.f;
        a.weight[row] = w;
      }
    }
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

}  // namespace

SNAP_DEBUG_READER(debug_flags_paged)

// ---------------------------------------------------------------- host side
PagedGeometry paged_geometry(const snap_params& p, int n, int max_rows, bool weigh) {
  PagedGeometry g{};
  const int units = (n > 0 ? n : 1) * p.n_kv_heads, G = p.n_q_heads / p.n_kv_heads;
  g.target = units < kItemTarget / 2 ? kItemTarget - units : kItemTarget / 2;
  const int64_t blocks = (int64_t)units * ((max_rows + kBlockRows - 1) / kBlockRows);
  // ceil(blocks / C) a unit, C >= blocks / target: at most target + units items,
  // and no more than there are blocks
  g.max_items = (int)(blocks < g.target + units ? blocks : g.target + units);
  size_t off = 0;
  g.off_part = off;
  off = align256(off + (size_t)g.max_items * G * p.d_v * sizeof(float));
  g.off_ml = off;
  off = align256(off + (size_t)g.max_items * G * sizeof(float2));
  g.off_z = off;
  if (weigh) off = align256(off + (size_t)blocks * kBlockRows * G * sizeof(float));
  g.bytes = off;
  return g;
}

snap_status launch_paged_append(const snap_params& p, const snap_paged_cache& c, const int32_t* rows,
                                const int32_t* pos, int n, const int32_t* slot_ids, const int32_t* lengths, int max_len,
                                const void* k_new, const int64_t* k_stride, const void* v_new, const int64_t* v_stride,
                                const float* weight_new, hipStream_t stream) {
  PagedAppendArgs a = {};
  a.k_new = k_new;
  a.v_new = p.v_in_k ? nullptr : v_new;
  a.weight_new = weight_new;
  a.ck = c.k;
  a.cv = p.v_in_k ? nullptr : c.v;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.token = c.token;
  a.weight = c.weight;
  a.rows = rows;
  a.pos = pos;
  a.slot_ids = slot_ids;
  a.lengths = lengths;
  a.table = c.page_table;
  a.Hkv = p.n_kv_heads;
  a.dk = p.d_qk;
  a.dv = p.d_v;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = log2_of(c.page_size);
  a.max_pages = c.max_pages;
  a.max_len = max_len;
  const int64_t kd[3] = {(int64_t)p.n_kv_heads * max_len * p.d_qk, (int64_t)max_len * p.d_qk, p.d_qk};
  const int64_t vd[3] = {(int64_t)p.n_kv_heads * max_len * p.d_v, (int64_t)max_len * p.d_v, p.d_v};
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = k_stride ? k_stride[i] : kd[i];
    a.vs[i] = v_stride ? v_stride[i] : vd[i];
  }
  const dim3 grid((max_len + kAppendTokens - 1) / kAppendTokens, p.n_kv_heads, n);
  if (p.kv_dtype == SNAP_FP8_E4M3)
    hipLaunchKernelGGL((paged_append<uint16_t, uint8_t>), grid, dim3(256), 0, stream, a);
  else if (p.kv_dtype == SNAP_BF16)
    hipLaunchKernelGGL((paged_append<uint16_t, uint16_t>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_append<float, float>), grid, dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

snap_status launch_paged_decode(const snap_params& p, const snap_paged_cache& c, const int32_t* rows,
                                const int32_t* pos, int n, const int32_t* slot_ids, int max_rows, const void* q,
                                const void* k_new, const void* v_new, void* out, int out_dtype, bool weigh, void* ws,
                                hipStream_t stream) {
  if (k_new) {
    const snap_status st = launch_paged_append(p, c, rows, pos, n, slot_ids, nullptr, 1, k_new, nullptr, v_new, nullptr,
                                               nullptr, stream);
    if (st != SNAP_OK) return st;
  }
  const PagedGeometry geo = paged_geometry(p, n, max_rows, weigh);
  PagedArgs a = {};
  a.q = q;
  a.ck = c.k;
  a.cv = p.v_in_k ? nullptr : c.v;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.rows = rows;
  a.slot_ids = slot_ids;
  a.table = c.page_table;
  a.part = (float*)((unsigned char*)ws + geo.off_part);
  a.ml = (float2*)((unsigned char*)ws + geo.off_ml);
  a.z = weigh ? (float*)((unsigned char*)ws + geo.off_z) : nullptr;
  a.weight = c.weight;
  a.out = out;
  a.n = n;
  a.Hq = p.n_q_heads;
  a.Hkv = p.n_kv_heads;
  a.G = p.n_q_heads / p.n_kv_heads;
  a.dk = p.d_qk;
  a.dv = p.d_v;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = log2_of(c.page_size);
  a.max_pages = c.max_pages;
  a.max_rows = max_rows;
  a.target = geo.target;
  a.max_items = geo.max_items;
  a.out_bf16 = out_dtype == SNAP_BF16;
  a.q_f32 = p.in_dtype == SNAP_F32;
  a.scale = p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_qk);
  const dim3 grid(geo.max_items, a.G);
  if (p.kv_dtype == SNAP_F32)
    hipLaunchKernelGGL((paged_decode<float>), grid, dim3(64), 0, stream, a);
  else if (p.kv_dtype == SNAP_BF16)
    hipLaunchKernelGGL((paged_decode<uint16_t>), grid, dim3(64), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_decode<uint8_t>), grid, dim3(64), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  hipLaunchKernelGGL(paged_join, dim3(n * p.n_q_heads), dim3(64), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  if (weigh) {
    hipLaunchKernelGGL(paged_weigh, dim3((max_rows + 255) / 256, n * p.n_kv_heads), dim3(256), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  }
  return SNAP_OK;
}

}  // namespace snap
