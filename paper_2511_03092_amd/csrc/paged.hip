// paged.hip -- the paged cache: storing new tokens, and attention of one new
// token per sequence over every row its slot holds.
//
//   paged_append   stores the tokens of a prompt or of a step
//   paged_gqa      64- and 128-wide rows: one wave per work item on the matrix
//                  units; a step's new token is stored in the same launch
//   paged_decode   latent rows: one wave per (work item, query head)
//   paged_join     merges the items of a (sequence, query head) -> out, and adds
//                  the rows' softmax weights to their accumulated ones
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
// with the SNAP_KV_AUTO hint, calls of at least this many cache bytes (at
// max_rows) read with streaming loads: half the 256 MB last-level cache
constexpr size_t kStreamingCallBytes = (size_t)128 << 20;

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
  // a step: the token to store at row rows[slot] before it is attended, [n][Hkv][dk]
  // / [n][Hkv][dv]; NULL when the launch only attends
  const void* k_new;
  const void* v_new;
  const int32_t* pos;
  int32_t* token;
  int n, Hq, Hkv, G, dk, dv, n_slots, n_pages, page_shift, max_pages, max_rows, target, max_items, out_bf16;
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
  if constexpr (sizeof(KV) == 2)
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
      q[i] = bf16_bits_to_f32(((const uint16_t*)a.q)[qo + i * 64 + lane]);
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

// ---------------------------------------------------------------- 64- and 128-wide rows
// One wave per work item, for the G query heads of its KV head at once: a block
// of 32 rows against the heads (padded to 16 columns) on the matrix units, an
// online softmax in the exp2 domain, the probabilities times the values on the
// matrix units.  Lane (l16, lg) holds head l16's logits of rows 4 lg + e of each
// 16-row half, which is also what the second product takes from it, so they
// never leave the lane; its keys are 16 bytes at byte 64 j + 16 lg of row l16,
// one load instruction reading 64 contiguous bytes of each of 16 rows; its values
// are the D / 16 dims from (D / 16) l16 of eight rows.
// A half lies in one page (pages hold 16 rows or more).  The wave keeps the ids of
// 64 pages, one a lane, and takes each half's by a lane read, so no load waits on
// a page table.
// A head's reference maximum moves only when a block's exceeds it by kStaleMax
// (log2 units), so the accumulators are rescaled on few blocks.
// 16-bit and fp8 rows: probabilities enter the products as two bf16 terms of 8
// bits each, truncated: off by under 2^-16 relative.  One term would be off by up
// to 2^-8, which the heaviest rows of a head show in the output; the second costs
// D / 16 matrix instructions a block, which the loads hide.  fp32 rows: fp32
// matrix instructions throughout.
constexpr float kStaleMax = 8.f;
enum { kKvBf16 = 0, kKvFp8 = 1, kKvF32 = 2 };

template <bool NT, typename T>
__device__ __forceinline__ T load_as(const void* p) {
  if constexpr (NT)
    return __builtin_nontemporal_load((const T*)p);
  else
    return *(const T*)p;
}

// 8 E4M3 codes -> 8 bf16 (exact)
__device__ __forceinline__ u32x4 codes_to_bf16(uint32_t c0, uint32_t c1) {
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.0f, false));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.0f, true));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.0f, false));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.0f, true));
  return o;
}

// 8 bf16 -> the 8 E4M3 codes of value / scale, as the append stores them
__device__ __forceinline__ u32x2 bf16_to_codes(u32x4 raw, float scale) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_bits_to_f32(raw[i] & 0xffffu) / scale;
    f[2 * i + 1] = bf16_bits_to_f32(raw[i] >> 16) / scale;
  }
  return u32x2{e4m3x4_hw(f[0], f[1], f[2], f[3]), e4m3x4_hw(f[4], f[5], f[6], f[7])};
}

// The ids of 64 pages of a slot from page `first` on, one a lane.
struct PageIds {
  int first, id;
  __device__ __forceinline__ void load(const PagedArgs& a, int slot, int page) {
    first = page;
    const int p = page + (tid() & 63);
    id = p < a.max_pages ? a.table[(size_t)slot * a.max_pages + p] : -1;
  }
  // index of row r (wave-uniform, never before the last one asked for) among the
  // rows of all pages, or -1
  __device__ __forceinline__ int64_t row(const PagedArgs& a, int slot, int g, int r) {
    const int page = r >> a.page_shift;
    if (page - first >= 64) load(a, slot, page);
    const int id_r = __builtin_amdgcn_readlane(id, page - first);
    if (id_r < 0 || id_r >= a.n_pages) return -1;
    return (((int64_t)id_r * a.Hkv + g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
  }
};

// This item's place: unit (s, g), rows [r0, r1), and the new token's row when it
// is this item's to store (-1 otherwise).
struct PagedItem {
  PagedSeq s;
  int g, r0, r1, rnew;
};
__device__ __forceinline__ bool paged_item(const PagedArgs& a, int item, PagedItem& it) {
  if (!paged_seq(a, item, true, it.s)) return false;
  if (!debug_check(item < a.max_items, kDbgPagedItem)) return false;
  const int local = item - it.s.item0, chunk = local % it.s.items;
  it.g = local / it.s.items;
  it.r0 = (int)((int64_t)chunk * it.s.blocks / it.s.items) * kBlockRows;
  it.r1 = min(it.s.len, (int)((int64_t)(chunk + 1) * it.s.blocks / it.s.items) * kBlockRows);
  it.rnew = a.k_new && chunk == it.s.items - 1 ? uniform(a.rows[it.s.slot]) : -1;
  return true;
}

template <int D, int KV, bool NT>
__global__ __launch_bounds__(64) void paged_gqa(PagedArgs a) {
  constexpr int E = KV == kKvFp8 ? 1 : (KV == kKvBf16 ? 2 : 4);  // bytes of an element
  constexpr int NK = D * E / 64;                                 // key loads a half
  constexpr int VE = D / 16;                                     // value dims a lane
  constexpr int NQ = KV == kKvFp8 ? 2 * NK : NK;                 // query pieces
  constexpr int NF = KV == kKvF32 ? VE : 1;
  typedef uint32_t VRaw __attribute__((ext_vector_type(VE * E / 4)));
  const int lane = tid(), l16 = lane & 15, lg = lane >> 4, item = bid_x();
  PagedItem it;
  if (!paged_item(a, item, it)) return;
  const int slot = it.s.slot, g = it.g, r0 = it.r0, r1 = it.r1, b = it.s.b;
  PageIds pages;
  pages.load(a, slot, r0 >> a.page_shift);
  const bool hval = l16 < a.G;
  const unsigned char* kbase = (const unsigned char*)a.ck;
  const unsigned char* vbase = a.cv ? (const unsigned char*)a.cv : kbase;
  u32x4 q[NQ];
  {
    constexpr int QE = KV == kKvF32 ? 4 : 2;
    const unsigned char* qp = (const unsigned char*)a.q + ((size_t)b * a.Hq + g * a.G + (hval ? l16 : 0)) * D * QE;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      // the dims of the lane's key piece (fp8: of each half of it)
      const int off = KV == kKvFp8 ? (64 * (j / 2) + 16 * lg + 8 * (j & 1)) * 2 : 64 * j + 16 * lg;
      q[j] = hval ? *(const u32x4*)(qp + off) : u32x4{0u, 0u, 0u, 0u};
    }
  }
  const float ksc = KV == kKvFp8 ? a.k_scale[(size_t)slot * a.Hkv + g] : 1.f;
  const float vsc = KV == kKvFp8 ? (a.cv ? a.v_scale : a.k_scale)[(size_t)slot * a.Hkv + g] : 1.f;
  const float xs = a.scale * kLog2e * ksc;
  // the new token's row in the cache's form: pieces of its input (fp8: the codes,
  // quantised once into LDS, keys in [0, D), values after them)
  __shared__ __align__(16) unsigned char newq[KV == kKvFp8 ? 2 * D : 16];
  const unsigned char* knew = nullptr;
  const unsigned char* vnew = nullptr;
  if (it.rnew >= 0) {
    const size_t u = (size_t)b * a.Hkv + g;
    knew = (const unsigned char*)a.k_new + u * D * (KV == kKvFp8 ? 2 : E);
    vnew = a.cv ? (const unsigned char*)a.v_new + u * D * (KV == kKvFp8 ? 2 : E) : knew;
    if constexpr (KV == kKvFp8) {
      constexpr int kc = D / 8;
      if (lane < kc)
        *(u32x2*)(newq + 8 * lane) = bf16_to_codes(*(const u32x4*)(knew + 16 * lane), ksc);
      else if (lane < 2 * kc)
        *(u32x2*)(newq + 8 * lane) = bf16_to_codes(*(const u32x4*)(vnew + 16 * (lane - kc)), vsc);
      knew = newq;
      vnew = newq + D;
      __syncthreads();
    }
  }

  auto load_k = [&](int vb, int64_t h0, int64_t h1, u32x4* k0, u32x4* k1) {
    const bool plain = vb + 32 <= r1 && h0 >= 0 && h1 >= 0 && (it.rnew < vb || it.rnew >= vb + 32);
    const unsigned char* p0 = kbase + (size_t)h0 * (D * E) + l16 * (D * E) + 16 * lg;
    const unsigned char* p1 = kbase + (size_t)h1 * (D * E) + l16 * (D * E) + 16 * lg;
    if (plain) {
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        k0[j] = load_as<NT, u32x4>(p0 + 64 * j);
        k1[j] = load_as<NT, u32x4>(p1 + 64 * j);
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      k0[j] = k1[j] = u32x4{0u, 0u, 0u, 0u};
      if (h0 >= 0 && vb + l16 < r1) k0[j] = vb + l16 == it.rnew ? *(const u32x4*)(knew + 16 * lg + 64 * j) : load_as<NT, u32x4>(p0 + 64 * j);
      if (h1 >= 0 && vb + 16 + l16 < r1)
        k1[j] = vb + 16 + l16 == it.rnew ? *(const u32x4*)(knew + 16 * lg + 64 * j) : load_as<NT, u32x4>(p1 + 64 * j);
    }
  };

  float m = -INFINITY, mref = 0.f, lsum = 0.f;  // reference maximum (log2 units), its finite stand-in, sum
  f32x4 acc[VE];
#pragma unroll
  for (int c = 0; c < VE; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float* z = a.z && hval
                 ? a.z + ((it.s.block0 + (int64_t)g * it.s.blocks) * a.G + (int64_t)l16 * it.s.blocks) * kBlockRows + 4 * lg
                 : nullptr;

  u32x4 k0[NK], k1[NK];
  int64_t h0 = pages.row(a, slot, g, r0), h1 = r0 + 16 < r1 ? pages.row(a, slot, g, r0 + 16) : -1;
  load_k(r0, h0, h1, k0, k1);
  for (int vb = r0; vb < r1; vb += 32) {
    // values of this block, then keys of the next: the second product waits for
    // the values only
    VRaw v[8];
    const bool whole = vb + 32 <= r1 && h0 >= 0 && h1 >= 0;
    if (whole && (it.rnew < vb || it.rnew >= vb + 32)) {
      const unsigned char* p0 = vbase + ((size_t)h0 + 4 * lg) * (D * E) + l16 * (VE * E);
      const unsigned char* p1 = vbase + ((size_t)h1 + 4 * lg) * (D * E) + l16 * (VE * E);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = load_as<NT, VRaw>((i < 4 ? p0 : p1) + (i & 3) * (D * E));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = vb + (i < 4 ? 0 : 16) + 4 * lg + (i & 3);
        const int64_t hb = i < 4 ? h0 : h1;
        v[i] = VRaw{};
        if (hb >= 0 && r < r1)
          v[i] = r == it.rnew ? *(const VRaw*)(vnew + l16 * (VE * E))
                              : load_as<NT, VRaw>(vbase + ((size_t)hb + 4 * lg + (i & 3)) * (D * E) + l16 * (VE * E));
      }
    }
    u32x4 n0[NK], n1[NK];
    int64_t nh0 = -1, nh1 = -1;
    if (vb + 32 < r1) {
      nh0 = pages.row(a, slot, g, vb + 32);
      nh1 = vb + 48 < r1 ? pages.row(a, slot, g, vb + 48) : -1;
      load_k(vb + 32, nh0, nh1, n0, n1);
    }

    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      if constexpr (KV == kKvBf16) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k0[j]), __builtin_bit_cast(bf16x8, q[j]), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k1[j]), __builtin_bit_cast(bf16x8, q[j]), s1, 0, 0, 0);
      } else if constexpr (KV == kKvFp8) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 qq = __builtin_bit_cast(bf16x8, q[2 * j + u]);
          s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, codes_to_bf16(k0[j][2 * u], k0[j][2 * u + 1])), qq, s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, codes_to_bf16(k1[j][2 * u], k1[j][2 * u + 1])), qq, s1, 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float qq = __uint_as_float(q[j][u]);
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k0[j][u]), qq, s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k1[j][u]), qq, s1, 0, 0, 0);
        }
      }
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = s0[e];
      x[4 + e] = s1[e];
      if (!whole) {
        if (h0 < 0 || vb + 4 * lg + e >= r1) x[e] = -INFINITY;
        if (h1 < 0 || vb + 16 + 4 * lg + e >= r1) x[4 + e] = -INFINITY;
      }
    }
    if (z) {
      *(f32x4*)(z + vb) = f32x4{x[0], x[1], x[2], x[3]} * xs;
      *(f32x4*)(z + vb + 16) = f32x4{x[4], x[5], x[6], x[7]} * xs;
    }
    float bm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    bm = fmaxf(bm, __shfl_xor(bm, 16));
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    bm *= xs;
    const bool up = bm > m + kStaleMax;  // always for the first block with a row (m = -inf)
    if (wave_any(up)) {
      const float mnew = up ? bm : m;
      const float alpha = up ? fast_exp2(m - mnew) : 1.f;
#pragma unroll
      for (int c = 0; c < VE; ++c) acc[c] *= alpha;
      lsum *= alpha;
      m = mnew;
      mref = m == -INFINITY ? 0.f : m;  // no row yet: every x is -inf, exp2 gives 0
    }
    float pe[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) pe[i] = fast_exp2(fmaf(x[i], xs, -mref));
    lsum += ((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]));
    if constexpr (KV == kKvF32) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < NF; ++c)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][c]), pe[i], acc[c], 0, 0, 0);
    } else {
      // the second term is kept off zero (2^-126), so that an infinite value
      // times it stays infinite, as with the whole probability
      bf16x8 p[2];
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        u32x4 pw;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = part ? fmaxf(pe[2 * i], 0x1p-126f) : pe[2 * i];
          const float hi = part ? fmaxf(pe[2 * i + 1], 0x1p-126f) : pe[2 * i + 1];
          pe[2 * i] -= __uint_as_float(__float_as_uint(pe[2 * i]) & 0xffff0000u);
          pe[2 * i + 1] -= __uint_as_float(__float_as_uint(pe[2 * i + 1]) & 0xffff0000u);
          pw[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
        p[part] = __builtin_bit_cast(bf16x8, pw);
      }
      uint32_t vw[8][VE / 2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (KV == kKvBf16) {
#pragma unroll
          for (int u = 0; u < VE / 2; ++u) vw[i][u] = v[i][u];
        } else {
#pragma unroll
          for (int u = 0; u < VE / 4; ++u) {
            vw[i][2 * u] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i][u], 1.0f, false));
            vw[i][2 * u + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i][u], 1.0f, true));
          }
        }
      }
#pragma unroll
      for (int c = 0; c < VE; ++c) {
        const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
        u32x4 av;
#pragma unroll
        for (int i = 0; i < 4; ++i) av[i] = __builtin_amdgcn_perm(vw[2 * i + 1][c >> 1], vw[2 * i][c >> 1], sel);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), p[1], acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), p[0], acc[c], 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      k0[j] = n0[j];
      k1[j] = n1[j];
    }
    h0 = nh0;
    h1 = nh1;
  }
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  // the new row: no other item reads it
  if (it.rnew >= 0 && it.rnew < (a.max_pages << a.page_shift)) {
    const int64_t row = paged_row(a, slot, g, it.rnew);
    if (row >= 0) {
      constexpr int kp = D * E / 16;  // pieces of a row
      if (lane < kp)
        *(u32x4*)((unsigned char*)const_cast<void*>(a.ck) + row * (D * E) + 16 * lane) = *(const u32x4*)(knew + 16 * lane);
      else if (a.cv && lane < 2 * kp)
        *(u32x4*)((unsigned char*)const_cast<void*>(a.cv) + row * (D * E) + 16 * (lane - kp)) =
            *(const u32x4*)(vnew + 16 * (lane - kp));
      if (lane == 0 && a.token) a.token[row] = a.pos[slot];
      if (lane == 0 && a.weight) a.weight[row] = 0.f;
    }
  }
  if (!hval) return;
  const size_t pi = (size_t)item * a.G + l16;
  if (lg == 0) a.ml[pi] = make_float2(m, lsum);
  float* dst = a.part + pi * D + 4 * lg * VE;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int c = 0; c < VE; c += 4)
      *(f32x4*)(dst + e * VE + c) = f32x4{acc[c][e], acc[c + 1][e], acc[c + 2][e], acc[c + 3][e]} * vsc;
}

// ---------------------------------------------------------------- join
// One launch merges the items of every (sequence, query head) into its output
// and, with weights, adds the softmax weights of the rows to theirs.  Workgroups
// [0, n Hq slices) merge, a slice of DV value dims each: thread t takes dims 4 (t
// % DG) .. + 3 of items t / DG, t / DG + CL, ...  The others take one work item's
// rows each (of equal length whatever their sequence, as in the attention), four
// rows a thread, after the references and sums of the unit's G heads.
constexpr int kJoinThreads = 256;

// The largest reference and the sum of a unit's items for head h of it, by a wave.
__device__ __forceinline__ float2 joined_ml(const PagedArgs& a, const PagedSeq& s, int g, int h) {
  const float2* ml = a.ml + (size_t)(s.item0 + g * s.items) * a.G + h;
  const int lane = tid() & 63;
  float m = -INFINITY, l = 0.f;
  for (int i = lane; i < s.items; i += 64) {
    const float2 v = ml[(size_t)i * a.G];
    const float mn = fmaxf(m, v.x);
    if (mn != -INFINITY) l = l * fast_exp2(m - mn) + v.y * fast_exp2(v.x - mn);
    m = mn;
  }
  float M = m;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
  return make_float2(M, warp_sum(m == -INFINITY ? 0.f : l * fast_exp2(m - M)));
}

template <int DV>
__global__ __launch_bounds__(kJoinThreads) void paged_join(PagedArgs a, int merges) {
  constexpr int DG = DV / 4, CL = kJoinThreads / DG;
  __shared__ f32x4 sacc[kJoinThreads];
  __shared__ float2 sml[16];
  const int t = tid(), w = uniform(t >> 6);
  if (bid_x() < merges) {
    const int slices = a.dv / DV, sl = bid_x() % slices, bh = bid_x() / slices;
    const int b = bh / a.Hq, qh = bh % a.Hq, g = qh / a.G, h = qh % a.G;
    PagedSeq s;
    if (!paged_seq(a, b, false, s) || s.slot < 0 || s.slot >= a.n_slots) return;
    const float2 ml = joined_ml(a, s, g, h);
    const int dg = t % DG, cl = t / DG;
    const size_t p0 = (size_t)(s.item0 + g * s.items) * a.G + h;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = cl; i < s.items; i += CL) {
      const size_t pi = p0 + (size_t)i * a.G;
      const float mi = a.ml[pi].x;
      const f32x4 v = *(const f32x4*)(a.part + pi * a.dv + sl * DV + 4 * dg);
      // an item none of whose rows is there has accumulated zeros
      o += v * (mi == -INFINITY ? 0.f : fast_exp2(mi - ml.x));
    }
    sacc[t] = o;
    __syncthreads();
    if (cl) return;
#pragma unroll
    for (int c = 1; c < CL; ++c) o += sacc[dg + DG * c];
    o *= ml.y > 0.f ? 1.f / ml.y : 0.f;
    const size_t oi = (size_t)bh * a.dv + sl * DV + 4 * dg;
    if (a.out_bf16)
      *(u32x2*)((uint16_t*)a.out + oi) = u32x2{f32_to_bf16_bits(o[0]) | (f32_to_bf16_bits(o[1]) << 16),
                                               f32_to_bf16_bits(o[2]) | (f32_to_bf16_bits(o[3]) << 16)};
    else
      *(f32x4*)((float*)a.out + oi) = o;
    return;
  }
  PagedItem it;
  if (!paged_item(a, bid_x() - merges, it)) return;
  for (int h = w; h < a.G; h += kJoinThreads / 64) {
    const float2 ml = joined_ml(a, it.s, it.g, h);
    if ((t & 63) == 0) sml[h] = make_float2(ml.x, ml.y > 0.f ? 1.f / ml.y : 0.f);
  }
  __syncthreads();
  const float* z = a.z + (it.s.block0 + (int64_t)it.g * it.s.blocks) * a.G * kBlockRows;
  for (int r = it.r0 + 4 * t; r < it.r1; r += 4 * kJoinThreads) {
    const int64_t row = paged_row(a, it.s.slot, it.g, r);  // four rows of one page
    if (row < 0) continue;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int h = 0; h < a.G; ++h) {
      const f32x4 y = *(const f32x4*)(z + (int64_t)h * it.s.blocks * kBlockRows + r);
      const float2 ml = sml[h];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(fast_exp2(y[e] - ml.x), ml.y, sum[e]);
    }
    if (r + 4 <= it.r1) {
      f32x4* p = (f32x4*)(a.weight + row);
      *p = *p + sum;
    } else {
      for (int e = 0; r + e < it.r1; ++e) a.weight[row + e] += sum[e];
    }
  }
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
  const bool gqa = p.d_qk == p.d_v;
  if (k_new && !gqa) {
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
  a.scale = p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_qk);
  const size_t elt = p.kv_dtype == SNAP_F32 ? 4 : (p.kv_dtype == SNAP_BF16 ? 2 : 1);
  const size_t call_bytes = (size_t)n * p.n_kv_heads * max_rows * (p.d_qk + (p.v_in_k ? 0 : p.d_v)) * elt;
  const bool nt = p.kv_reuse == SNAP_KV_STREAM || (p.kv_reuse == SNAP_KV_AUTO && call_bytes >= kStreamingCallBytes);
  if (gqa) {
    a.k_new = k_new;
    a.v_new = v_new;
    a.pos = pos;
    a.token = c.token;
    void (*k)(PagedArgs);
    if (p.d_qk == 64)
      k = p.kv_dtype == SNAP_F32    ? (nt ? paged_gqa<64, kKvF32, true> : paged_gqa<64, kKvF32, false>)
          : p.kv_dtype == SNAP_BF16 ? (nt ? paged_gqa<64, kKvBf16, true> : paged_gqa<64, kKvBf16, false>)
                                    : (nt ? paged_gqa<64, kKvFp8, true> : paged_gqa<64, kKvFp8, false>);
    else
      k = p.kv_dtype == SNAP_F32    ? (nt ? paged_gqa<128, kKvF32, true> : paged_gqa<128, kKvF32, false>)
          : p.kv_dtype == SNAP_BF16 ? (nt ? paged_gqa<128, kKvBf16, true> : paged_gqa<128, kKvBf16, false>)
                                    : (nt ? paged_gqa<128, kKvFp8, true> : paged_gqa<128, kKvFp8, false>);
    hipLaunchKernelGGL(k, dim3(geo.max_items), dim3(64), 0, stream, a);
  } else {
    const dim3 grid(geo.max_items, a.G);
    if (p.kv_dtype == SNAP_BF16)
      hipLaunchKernelGGL((paged_decode<uint16_t>), grid, dim3(64), 0, stream, a);
    else
      hipLaunchKernelGGL((paged_decode<uint8_t>), grid, dim3(64), 0, stream, a);
  }
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  const int merges = n * p.n_q_heads * (p.d_v == 512 ? 4 : 1);
  const dim3 join(merges + (weigh ? geo.max_items : 0));
  if (p.d_v == 64)
    hipLaunchKernelGGL(paged_join<64>, join, dim3(kJoinThreads), 0, stream, a, merges);
  else  // 512-wide values: 128-dim slices
    hipLaunchKernelGGL(paged_join<128>, join, dim3(kJoinThreads), 0, stream, a, merges);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  return SNAP_OK;
}

}  // namespace snap
