// paged.hip -- the paged cache: storing new tokens, and attention of one new
// token per sequence over every row its slot holds.
//
//   paged_append   stores the tokens of a prompt or of a step (paged_append_mapped: of
//                  a packed batch, by its map)
//   paged_gqa      64- and 128-wide rows: one wave per work item on the matrix
//                  units
//   paged_latent   latent rows: four waves per work item, through LDS
//   paged_join     merges the items of a (sequence, query head) -> out, and adds
//                  the rows' softmax weights to their accumulated ones
// A step's new token is stored in the attention launch, by the item that ends
// with it, which reads it from its input.
//
// Work items.  Sequences are of unequal length and their lengths are on the
// device, so the rows are cut there: every unit (sequence, KV head) takes
// ceil(blocks / C) items of nearly equal length, C the 32-row blocks of all
// units over the items wanted, so that an item is as long as another whatever
// sequence it is of.  Every wave finds its item from the lengths alone (very many
// short units are not cut).
#include <math.h>

#include "lds_dma.h"
#include "snap_internal.h"

namespace snap {

namespace {

constexpr int kBlockRows = 32;  // rows of a block
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
  float* z;      // logits in log2 units, [unit][its blocks][G][32 rows]; NULL without weights
  float* weight;
  void* out;
  // a step: the token to store at row rows[slot] before it is attended, [n][Hkv][dk]
  // / [n][Hkv][dv]; NULL when the launch only attends
  const void* k_new;
  const void* v_new;
  const int32_t* pos;
  int32_t* token;
  int n, Hq, Hkv, G, dk, dv, n_slots, n_pages, page_shift, max_pages, max_rows, waves, target, max_items, whole, out_bf16;
  float scale2, scale2_lo;  // scale * log2(e) in two terms, both > 0
};

// The rows sequence b attends (0 for a slot id out of range).
__device__ __forceinline__ int rows_of(const PagedArgs& a, int b, int& slot) {
  slot = a.slot_ids[b];
  const bool ok = slot >= 0 && slot < a.n_slots;
  const int r = a.rows[ok ? slot : 0];  // no branch: the loads of several sequences go out together
  return !ok || r < 0 ? 0 : (r >= a.max_rows ? a.max_rows : r + 1);
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
  if (a.whole) {  // item i is unit i
    s.b = by_item ? key / a.Hkv : key;
    if (s.b >= a.n) return false;
    int slot;
    s.len = uniform(rows_of(a, s.b, slot));
    s.slot = uniform(slot);
    s.blocks = (s.len + kBlockRows - 1) / kBlockRows;
    s.items = s.blocks > 0;
    s.item0 = s.b * a.Hkv;
    s.block0 = (int64_t)s.item0 * ((a.max_rows + kBlockRows - 1) / kBlockRows);
    return !by_item || s.items;
  }
  int64_t mine = 0;
  int nb0 = 0;
#pragma unroll 4
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    int slot;
    const int b = b0 + lane, len = rows_of(a, min(b, a.n - 1), slot);
    const int nb = b < a.n ? (len + kBlockRows - 1) / kBlockRows : 0;
    if (b0 == 0) nb0 = nb;
    mine += nb;
  }
  const int64_t total = wave_total((int)(mine & 0xfffff)) + ((int64_t)wave_total((int)(mine >> 20)) << 20);
  const int C = paged_chunk(a.waves, a.target, a.n, a.Hkv, total,
                            [&](int c) { return wave_total(c > 0 ? (nb0 + c - 1) / c : 0); });  // (up to 64 sequences)
  int items_before = 0, slot_next;
  int64_t blocks_before = 0;
  int len_next = rows_of(a, min(lane, a.n - 1), slot_next);
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    const int b = b0 + lane, slot = slot_next, len = b < a.n ? len_next : 0;
    if (b0 + 64 < a.n) len_next = rows_of(a, min(b + 64, a.n - 1), slot_next);  // while this one is counted
    const int nb = (len + kBlockRows - 1) / kBlockRows;
    const int ni = (nb + C - 1) / C;
    const int si = wave_scan(ni), sb = wave_scan(nb);
    const int first = items_before + a.Hkv * (si - ni);
    const bool here = b < a.n && (by_item ? key >= first && key < first + a.Hkv * ni : key == b);
    const uint64_t m = __builtin_amdgcn_ballot_w64(here);
    if (m) {
      const int at = __builtin_ctzll(m);
      s.b = b0 + at;
      s.slot = __builtin_amdgcn_readlane(slot, at);
      s.len = __builtin_amdgcn_readlane(len, at);
      s.blocks = __builtin_amdgcn_readlane(nb, at);
      s.items = __builtin_amdgcn_readlane(ni, at);
      s.item0 = __builtin_amdgcn_readlane(first, at);
      s.block0 = blocks_before + (int64_t)a.Hkv * __builtin_amdgcn_readlane(sb - nb, at);
      // (items past the launch would be rows that nothing attends)
      return debug_check(s.item0 + a.Hkv * s.items <= a.max_items, kDbgPagedItem);
    }
    items_before += a.Hkv * __builtin_amdgcn_readlane(si, 63);
    blocks_before += (int64_t)a.Hkv * __builtin_amdgcn_readlane(sb, 63);
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
// HBM bound: 8 sequences of 19k to 128k rows x 8 KV heads, 128-wide bf16 (2.52 GB) 380
// to 397 us, 6.3 to 6.6 TB/s with the join; fp8 210 us, 6.0 TB/s.  Values prefetched a block ahead
// like the keys change nothing, there or for short sequences.
// 16-bit and fp8 rows: probabilities enter the products whole, as three bf16 terms
// of 8 bits.  Two terms, cut off, are off by up to 2^-15 and always to the same side,
// which fp32 outputs show and bf16 ones as roundings to the other neighbour; the third
// costs D / 16 matrix instructions a block, mostly hidden by the loads (128-wide fp8,
// 32 x 8 heads of up to 16384 rows with weights, 123 -> 126 us; bf16 none).  fp32 rows:
// fp32 matrix instructions throughout.
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

// Four products as logits in log2 units: the scale's second term keeps its rounding
// (6e-8 relative, 1e-6 of a probability whose logit is 16) out of them.  It is
// positive, so a masked product's -inf stays -inf.
__device__ __forceinline__ f32x4 logits4(const float* x, float xs, float xlo) {
  return f32x4{fmaf(x[0], xs, x[0] * xlo), fmaf(x[1], xs, x[1] * xlo), fmaf(x[2], xs, x[2] * xlo), fmaf(x[3], xs, x[3] * xlo)};
}

// Eight probabilities as three bf16 terms, whose sum they are (pe is used up).  The
// second and third are kept off zero (2^-126), so that an infinite value times them
// stays infinite, as with the whole probability.
__device__ __forceinline__ void three_terms(float (&pe)[8], bf16x8 (&p)[3]) {
#pragma unroll
  for (int part = 0; part < 3; ++part) {
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
}

// The same as two terms, each rounded to nearest: off by at most 2^-18 relative (half a
// step of half a step), to either side.
__device__ __forceinline__ void two_terms(float (&pe)[8], bf16x8 (&p)[2]) {
  u32x4 first, second;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    first[i] = pack_bf16x2(pe[2 * i], pe[2 * i + 1]);
    pe[2 * i] -= __uint_as_float(first[i] << 16);
    pe[2 * i + 1] -= __uint_as_float(first[i] & 0xffff0000u);
    second[i] = pack_bf16x2(pe[2 * i], pe[2 * i + 1]);
  }
  p[0] = __builtin_bit_cast(bf16x8, first);
  p[1] = __builtin_bit_cast(bf16x8, second);
}

// A loaded value is waited for here.  Before a loop, and behind a branch in one:
// where the compiler sees a load that may be in flight as the loop comes round, it
// waits at the value's use, every time, for all loads in flight.
template <typename T>
__device__ __forceinline__ void settle(T& v) {
  asm volatile("" : "+v"(v));
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
    if (page - first >= 64) {
      load(a, slot, page);
      settle(id);
    }
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
  const int local = item - it.s.item0, chunk = local % it.s.items;
  it.g = local / it.s.items;
  it.r0 = (int)((int64_t)chunk * it.s.blocks / it.s.items) * kBlockRows;
  it.r1 = min(it.s.len, (int)((int64_t)(chunk + 1) * it.s.blocks / it.s.items) * kBlockRows);
  it.rnew = a.k_new && chunk == it.s.items - 1 ? uniform(a.rows[it.s.slot]) : -1;
  return true;
}

// The share of wave w of `waves` that take unit `unit` together (none of the rows
// where there are fewer blocks); the last has the new token.  false: no such slot.
__device__ __forceinline__ bool paged_unit(const PagedArgs& a, int unit, int w, int waves, PagedItem& it) {
  it.s = {};
  it.s.b = unit / a.Hkv;
  it.g = unit % a.Hkv;
  int slot;
  it.s.len = uniform(rows_of(a, it.s.b, slot));
  it.s.slot = uniform(slot);
  if (it.s.slot < 0 || it.s.slot >= a.n_slots) return false;
  it.s.blocks = (it.s.len + kBlockRows - 1) / kBlockRows;
  it.r0 = min(it.s.len, w * it.s.blocks / waves * kBlockRows);
  it.r1 = min(it.s.len, (w + 1) * it.s.blocks / waves * kBlockRows);
  it.rnew = a.k_new && it.s.len > 0 && w == waves - 1 ? uniform(a.rows[it.s.slot]) : -1;
  return true;
}

// The weights of rows r .. r + 3, at index `row` of their page (-1: none), with the
// softmax weights of this call added, summed over the unit's heads in order; z: the
// unit's logits, ml: reference and 1 / sum of every head.  Row rnew had none yet.
__device__ __forceinline__ f32x4 new_weights(const PagedArgs& a, const float* z, const float2* ml, int64_t row, int r, int rnew) {
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (row < 0) return sum;
  f32x4 old = *(const f32x4*)(a.weight + row);
#pragma unroll 4
  for (int h = 0; h < a.G; ++h) {
    const f32x4 y = *(const f32x4*)(z + ((int64_t)(r / kBlockRows) * a.G + h) * kBlockRows + r % kBlockRows);
    const float2 m = ml[h];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(fast_exp2(y[e] - m.x), m.y, sum[e]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] += r + e == rnew ? 0.f : old[e];
  return sum;
}
// Stores them for the rows before `end`.
__device__ __forceinline__ void put_weights(const PagedArgs& a, int64_t row, int r, int end, f32x4 v) {
  if (row < 0) return;
  if (r + 4 <= end) {
    *(f32x4*)(a.weight + row) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e < end) a.weight[row + e] = v[e];
  }
}

// W: the logits go to the workspace, for the weights.  They are staged in LDS and
// leave in runs of 16 KB: writes between the streaming reads cost by their number
// more than by their bytes (8 sequences of 19k to 128k rows, 79 MB of logits beside
// 2.52 GB: 512-byte runs 527 us, 1 KB runs 510, 16 KB runs 455, none 392).  Eight
// waves a CU leave each 20 KB of LDS.
constexpr int kZStage = 4096;  // logits that are staged before they leave

// WAVES > 1: one workgroup takes a whole unit, each wave a share of its blocks, joins
// them in LDS, writes the output and adds the weights (whose logits stay in LDS): one
// launch instead of two, for calls so short that launches and dependent loads are
// most of them.
template <int D, int KV, bool NT, bool W, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void paged_gqa(PagedArgs a) {
  // WAVES == 1, W: kZStage logits and a block more; WAVES > 1: [WAVES / 2][G][D] for
  // the join, then, W, the unit's logits
  extern __shared__ __align__(16) float zstage[];
  constexpr int E = KV == kKvFp8 ? 1 : (KV == kKvBf16 ? 2 : 4);  // bytes of an element
  constexpr int NK = D * E / 64;                                 // key loads a half
  constexpr int VE = D / 16;                                     // value dims a lane
  constexpr int NQ = KV == kKvFp8 ? 2 * NK : NK;                 // query pieces
  constexpr int NF = KV == kKvF32 ? VE : 1;
  typedef uint32_t VRaw __attribute__((ext_vector_type(VE * E / 4)));
  const int lane = tid() & 63, w = WAVES == 1 ? 0 : uniform(tid() >> 6), l16 = lane & 15, lg = lane >> 4, item = bid_x();
  PagedItem it;
  if constexpr (WAVES == 1) {
    if (!paged_item(a, item, it)) return;
  } else {
    if (!paged_unit(a, item, w, WAVES, it)) return;
  }
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
  float xs = a.scale2 * ksc, xlo = fmaxf(a.scale2_lo * ksc, 1e-37f);
  settle(xs);
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
      asm volatile("" ::: "memory");  // one wave's LDS operations take effect in order
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
    // A lane whose row is not there reads row 0 of page 0 (its logit is masked), the
    // new token's its input: the address is chosen, not the load, so that all loads
    // of the block are in flight together.
    const int ra = vb + l16, rb = ra + 16;
    if (h0 < 0 || ra >= r1) p0 = kbase + 16 * lg;
    else if (KV != kKvFp8 && ra == it.rnew) p0 = knew + 16 * lg;
    if (h1 < 0 || rb >= r1) p1 = kbase + 16 * lg;
    else if (KV != kKvFp8 && rb == it.rnew) p1 = knew + 16 * lg;
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      k0[j] = load_as<NT, u32x4>(p0 + 64 * j);
      k1[j] = load_as<NT, u32x4>(p1 + 64 * j);
    }
  };

  float m = -INFINITY, mref = 0.f, lsum = 0.f;  // reference maximum (log2 units), its finite stand-in, sum
  f32x4 acc[VE];
#pragma unroll
  for (int c = 0; c < VE; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float* zunit = zstage + (WAVES / 2) * a.G * D;  // WAVES > 1
  float* z = W && WAVES == 1 ? a.z + (it.s.block0 + (int64_t)g * it.s.blocks) * a.G * kBlockRows : nullptr;
  int zrow = r0;  // first row staged

#pragma unroll
  for (int j = 0; j < NQ; ++j) settle(q[j]);
  settle(pages.id);
  u32x4 k0[NK], k1[NK];
  int64_t h0 = r0 < r1 ? pages.row(a, slot, g, r0) : -1, h1 = r0 + 16 < r1 ? pages.row(a, slot, g, r0 + 16) : -1;
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
      for (int i = 0; i < 8; ++i) {  // as for the keys; a value whose row is not there is zeroed before its product
        const int r = vb + (i < 4 ? 0 : 16) + 4 * lg + (i & 3);
        const int64_t hb = i < 4 ? h0 : h1;
        const unsigned char* from = vbase + ((size_t)hb + 4 * lg + (i & 3)) * (D * E);
        if (hb < 0 || r >= r1) from = vbase;
        else if (KV != kKvFp8 && r == it.rnew) from = vnew;
        v[i] = load_as<NT, VRaw>(from + l16 * (VE * E));
      }
    }
    u32x4 n0[NK], n1[NK];
    int64_t nh0 = -1, nh1 = -1;
    if (vb + 32 < r1) {
      nh0 = pages.row(a, slot, g, vb + 32);
      nh1 = vb + 48 < r1 ? pages.row(a, slot, g, vb + 48) : -1;
      load_k(vb + 32, nh0, nh1, n0, n1);
    }

    const bool fresh = KV == kKvFp8 && it.rnew >= vb && it.rnew < min(r1, vb + 32);  // its codes are in LDS
    if (fresh) {
#pragma unroll
      for (int j = 0; j < NK; ++j) {
        const u32x4 c = *(const u32x4*)(newq + 16 * lg + 64 * j);
        k0[j] = vb + l16 == it.rnew ? c : k0[j];
        k1[j] = vb + 16 + l16 == it.rnew ? c : k1[j];
      }
    }
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f}, f0[4] = {}, f1[4] = {};
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
        for (int u = 0; u < 4; ++u) {  // four sums of D / 4 products: shorter chains of roundings
          const float qq = __uint_as_float(q[j][u]);
          f0[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k0[j][u]), qq, f0[u], 0, 0, 0);
          f1[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k1[j][u]), qq, f1[u], 0, 0, 0);
        }
      }
    }
    if constexpr (KV == kKvF32) {
      s0 = (f0[0] + f0[1]) + (f0[2] + f0[3]);
      s1 = (f1[0] + f1[1]) + (f1[2] + f1[3]);
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
    if constexpr (W) {
      if (hval) {
        float* st = (WAVES == 1 ? zstage + (vb - zrow) * a.G : zunit + vb * a.G) + l16 * kBlockRows + 4 * lg;
        *(f32x4*)st = logits4(x, xs, xlo);
        *(f32x4*)(st + 16) = logits4(x + 4, xs, xlo);
      }
      const int staged = (vb + 32 - zrow) * a.G;
      if (WAVES == 1 && (staged >= kZStage || vb + 32 >= r1)) {
        // one wave, whose LDS operations take effect in order: no barrier (which
        // would also wait for the loads in flight), only the compiler is held
        asm volatile("" ::: "memory");
        for (int i = 4 * lane; i < staged; i += 256) *(f32x4*)(z + (int64_t)zrow * a.G + i) = *(const f32x4*)(zstage + i);
        asm volatile("" ::: "memory");
        zrow = vb + 32;
      }
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
    for (int i = 0; i < 8; ++i) pe[i] = fast_exp2(fmaf(x[i], xs, fmaf(x[i], xlo, -mref)));
    lsum += ((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]));
    if (!whole || fresh) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = vb + (i < 4 ? 0 : 16) + 4 * lg + (i & 3);
        if ((i < 4 ? h0 : h1) < 0 || r >= r1) v[i] = VRaw{};
        else if (fresh && r == it.rnew) v[i] = *(const VRaw*)(newq + D + l16 * (VE * E));
      }
    }
    if constexpr (KV == kKvF32) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < NF; ++c)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][c]), pe[i], acc[c], 0, 0, 0);
    } else {
      bf16x8 p[3];
      three_terms(pe, p);
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
#pragma unroll
        for (int part = 2; part >= 0; --part)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), p[part], acc[c], 0, 0, 0);
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
      // (with weights a joined unit's first is written with the sum below)
      if (lane == 0 && a.weight && !(W && WAVES > 1 && it.rnew < r1)) a.weight[row] = 0.f;
    }
  }
  if constexpr (WAVES > 1) {
    __shared__ float2 mls[WAVES][16];
    __shared__ float2 joined[16];  // reference and 1 / sum of every head
    if (lg == 0) mls[w][l16] = make_float2(m, lsum);
    __syncthreads();
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) M = fmaxf(M, mls[i][l16].x);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float2 v = mls[i][l16];
      if (v.x != -INFINITY) L = fmaf(fast_exp2(v.x - M), v.y, L);
    }
    const float inv = L > 0.f ? 1.f / L : 0.f, f = m == -INFINITY ? 0.f : fast_exp2(m - M) * inv * vsc;
    if (w == 0 && lg == 0) joined[l16] = make_float2(M, inv);
#pragma unroll
    for (int c = 0; c < VE; ++c) acc[c] *= f;
    // the upper half of the waves hand theirs to the lower, until one has the sum
#pragma unroll
    for (int half = WAVES / 2; half >= 1; half /= 2) {
      float* to = zstage + ((w & (half - 1)) * a.G + l16) * D + 4 * lg * VE;
      if (w >= half && w < 2 * half && hval)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < VE; c += 4)
            *(f32x4*)(to + e * VE + c) = f32x4{acc[c][e], acc[c + 1][e], acc[c + 2][e], acc[c + 3][e]};
      __syncthreads();
      if (w < half && hval)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < VE; c += 4) {
            const f32x4 v = *(const f32x4*)(to + e * VE + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c + i][e] += v[i];
          }
      __syncthreads();
    }
    if (w == 0 && hval) {
      const size_t oi = ((size_t)b * a.Hq + g * a.G + l16) * D + 4 * lg * VE;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VE; c += 4) {
          if (a.out_bf16)
            *(u32x2*)((uint16_t*)a.out + oi + e * VE + c) =
                u32x2{pack_bf16x2(acc[c][e], acc[c + 1][e]), pack_bf16x2(acc[c + 2][e], acc[c + 3][e])};
          else
            *(f32x4*)((float*)a.out + oi + e * VE + c) = f32x4{acc[c][e], acc[c + 1][e], acc[c + 2][e], acc[c + 3][e]};
        }
    }
    if constexpr (W) {
      const int rnew = a.k_new ? uniform(a.rows[slot]) : -1;
      for (int r = 4 * tid(); r < it.s.len; r += 4 * 64 * WAVES) {
        const int64_t row = paged_row(a, slot, g, r);  // four rows of one page
        put_weights(a, row, r, it.s.len, new_weights(a, zunit, joined, row, r, rnew));
      }
    }
    return;
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

// ---------------------------------------------------------------- latent rows
// 576-wide rows whose first 512 dims are the values, bf16 or fp8.  Four waves per
// work item take blocks of 64 rows through two LDS stages of direct global -> LDS
// loads: wave w loads the rows [16w, 16w+16) of a block (in one page), forms their
// logits as soon as its own loads are there, and leaves them in LDS; after one
// barrier, which every wave reaches with its rows landed, each wave takes the
// softmax of all 64 rows and the value product for dims [128w, 128w+128).  So no
// key is read from LDS twice, no code converted twice for the same product, and a
// block needs two barriers: that one, and one before its stage is loaded again.
// A stage holds rows of CPR 16-byte pieces; piece c of row r sits at r CPR + (c ^
// swizzle(r)), within aligned groups of 8 (fp8: 4), which spreads both the key
// reads (one piece of 16 rows) and the value reads (16 pieces of a row) over the
// banks.  bf16 stages take 147 KB, one workgroup a CU; fp8 ones half, two.
// Rows past the sequence and in pages that are not there are loaded from a row of
// zeros: their probabilities are zero, and zero times whatever else might stand
// there need not be.
// Probabilities enter the value product as two bf16 terms rounded to nearest (2^-18):
// with one wave a SIMD nothing hides a third term's 16 matrix instructions a block (bf16
// 102.6 -> 107, fp8 72 -> 79 us in the cases below); against the same attention in fp32
// the bf16 outputs of the bf16 case are 9e-5 off with two terms, 7e-5 with three (mostly
// roundings to the other neighbour), 2e-4 with two that are cut off.
// HBM bound in bf16: 16 sequences of 32k rows (604 MB) 102 us, 5.9 TB/s; blocks of 32
// rows in four stages, the dims of a product split over the waves, take as long.  fp8
// (302 MB, 16 heads) 74 us: the conversions, and a block's two barriers with two
// workgroups a CU; the 32-row form takes 82.
constexpr int kLatRows = 64;
__device__ const u32x4 kZeroRow[72] = {};

template <bool FP8>
struct Lat {
  static constexpr int RB = FP8 ? 576 : 1152;  // bytes of a row
  static constexpr int CPR = RB / 16;
  static constexpr int NL = 16 * CPR / 64;     // loads a wave and block: 18 or 9
  static constexpr int Stage = kLatRows * RB;
  static __device__ __forceinline__ int swz(int r) { return (r >> 1) & (FP8 ? 3 : 7); }
  static __device__ __forceinline__ int at(int r, int c) { return (r * CPR + (c ^ swz(r))) * 16; }
};

typedef __attribute__((address_space(3))) void* lds_ptr;
// One wave-instruction of global -> LDS copy: lane i's 16 bytes land at lds + 16 i.
// In asm, so that the only order with later LDS reads is the explicit wait; M0
// (the LDS base) is saved and restored.
template <bool NT>
__device__ __forceinline__ void copy_to_lds(const void* from, const void* lds) {
  const uint32_t la = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)lds);
  uint32_t saved;
  if constexpr (NT)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off nt\n\ts_nop 0\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "s"(la), "v"(from) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_nop 0\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "s"(la), "v"(from) : "memory");
}

template <bool FP8, bool NT, bool W>
__global__ __launch_bounds__(256, FP8 ? 2 : 1) void paged_latent(PagedArgs a) {
  typedef Lat<FP8> L;
  constexpr int D = 576, DV = 512, XLd = kLatRows + 4;
  __shared__ __align__(16) unsigned char stage[2][L::Stage];
  __shared__ __align__(16) float xs_all[16 * XLd];  // a block's products by head
  const int lane = tid() & 63, w = uniform(tid() >> 6), l16 = lane & 15, lg = lane >> 4;
  PagedItem it;
  if (!paged_item(a, bid_x(), it)) return;
  const int slot = it.s.slot, g = it.g, r0 = it.r0, r1 = it.r1, b = it.s.b;
  PageIds pages;
  pages.load(a, slot, r0 >> a.page_shift);
  const bool hval = l16 < a.G;
  const unsigned char* cache = (const unsigned char*)a.ck;
  const unsigned char* knew = it.rnew >= 0 ? (const unsigned char*)a.k_new + ((size_t)b * a.Hkv + g) * (D * 2) : nullptr;
  const float ksc = FP8 ? a.k_scale[(size_t)slot * a.Hkv + g] : 1.f;
  const float xs = a.scale2 * ksc, xlo = fmaxf(a.scale2_lo * ksc, 1e-37f);
  // lane group lg feeds the piece 18 lg + t (fp8: half t % 2 of 9 lg + t / 2) of a
  // row to k-step t
  bf16x8 q[18];
  {
    const uint16_t* qp = (const uint16_t*)a.q + ((size_t)b * a.Hq + g * a.G + (hval ? l16 : 0)) * D;
#pragma unroll
    for (int t = 0; t < 18; ++t)
      q[t] = __builtin_bit_cast(bf16x8, hval ? *(const u32x4*)(qp + 8 * (18 * lg + t)) : u32x4{0u, 0u, 0u, 0u});
#pragma unroll
    for (int t = 0; t < 18; ++t) settle(q[t]);
    settle(pages.id);
  }
  int off[L::NL];  // this lane's pieces of a wave's 16 rows: bytes from their first
#pragma unroll
  for (int i = 0; i < L::NL; ++i) {
    const int sl = i * 64 + lane, r = sl / L::CPR;
    off[i] = r * L::RB + ((sl % L::CPR) ^ L::swz(r)) * 16;
  }
  int there = 0;  // bit s: the page of this wave's rows in stage s is there
  auto issue = [&](int blk) {
    const int vb = r0 + kLatRows * blk + 16 * w;
    unsigned char* dst = &stage[blk & 1][16 * w * L::RB];
    const int64_t base = vb < r1 ? pages.row(a, slot, g, vb) : -1;
    there = (there & ~(1 << (blk & 1))) | (base >= 0 ? 1 << (blk & 1) : 0);
    const unsigned char* rows = cache + (size_t)base * L::RB;
    if (base >= 0 && vb + 16 <= r1 && (it.rnew < vb || it.rnew >= vb + 16)) {
#pragma unroll
      for (int i = 0; i < L::NL; ++i) copy_to_lds<NT>(rows + off[i], dst + 1024 * i);
    } else {
#pragma unroll
      for (int i = 0; i < L::NL; ++i) {
        const int r = vb + off[i] / L::RB, piece = off[i] % L::RB;
        const unsigned char* from = rows + off[i];
        if (base < 0 || r >= r1) from = (const unsigned char*)kZeroRow + piece;
        else if (r == it.rnew) from = (FP8 ? (const unsigned char*)kZeroRow : knew) + piece;
        copy_to_lds<NT>(from, dst + 1024 * i);
      }
    }
  };

  float m = -INFINITY, mref = 0.f, lsum = 0.f;
  f32x4 acc[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float* z = W ? a.z + (it.s.block0 + (int64_t)g * it.s.blocks) * a.G * kBlockRows : nullptr;
  const int nblk = (r1 - r0 + kLatRows - 1) / kLatRows;
  issue(0);
  if (nblk > 1) issue(1);
  for (int i = 0; i < nblk; ++i) {
    // this wave's rows of block i have landed: only the next block's loads (and
    // what was issued after them) are in flight
    if (i + 1 < nblk)
      wait_vm<L::NL>();
    else
      wait_vm<0>();
    asm volatile("" ::: "memory");
    unsigned char* st = &stage[i & 1][0];
    const int vb = r0 + kLatRows * i, vw = vb + 16 * w;
    const bool have = (there >> (i & 1)) & 1;
    if constexpr (FP8) {
      if (have && it.rnew >= vw && it.rnew < min(r1, vw + 16) && lane < L::CPR) {  // the new row's codes, over the zeros
        const u32x4* src = (const u32x4*)knew + 2 * lane;
        const u32x2 c0 = bf16_to_codes(src[0], ksc), c1 = bf16_to_codes(src[1], ksc);
        *(u32x4*)(st + L::at(it.rnew - vb, lane)) = u32x4{c0[0], c0[1], c1[0], c1[1]};
      }
      asm volatile("" ::: "memory");
    }
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 18; t += FP8 ? 2 : 1) {
      const u32x4 k = *(const u32x4*)(st + L::at(16 * w + l16, FP8 ? 9 * lg + t / 2 : 18 * lg + t));
      if constexpr (FP8) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, codes_to_bf16(k[0], k[1])), q[t], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, codes_to_bf16(k[2], k[3])), q[t + 1], s, 0, 0, 0);
      } else {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), q[t], s, 0, 0, 0);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!have || vw + 4 * lg + e >= r1) s[e] = -INFINITY;
    *(f32x4*)(xs_all + l16 * XLd + 16 * w + 4 * lg) = s;
    lds_barrier();  // every wave's rows have landed and its products are there
    float x[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x4 v = *(const f32x4*)(xs_all + l16 * XLd + 16 * k + 4 * lg);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * k + e] = v[e];
    }
    if (W && w == 0 && hval) {
      float* zb = z + ((int64_t)(vb / kBlockRows) * a.G + l16) * kBlockRows + 4 * lg;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (vb + 16 * k < r1)
          *(f32x4*)(zb + (k >> 1) * a.G * kBlockRows + 16 * (k & 1)) = logits4(x + 4 * k, xs, xlo);
    }
    float bm = -INFINITY;
#pragma unroll
    for (int k = 0; k < 16; ++k) bm = fmaxf(bm, x[k]);
    bm = fmaxf(bm, __shfl_xor(bm, 16));
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    bm *= xs;
    const bool up = bm > m + kStaleMax;
    if (wave_any(up)) {
      const float mnew = up ? bm : m;
      const float alpha = up ? fast_exp2(m - mnew) : 1.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[c] *= alpha;
      lsum *= alpha;
      m = mnew;
      mref = m == -INFINITY ? 0.f : m;
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      float pe[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) pe[k] = fast_exp2(fmaf(x[8 * kk + k], xs, fmaf(x[8 * kk + k], xlo, -mref)));
      lsum += ((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]));
      bf16x8 p[2];
      two_terms(pe, p);
      u32x4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int r = 32 * kk + (k < 4 ? 0 : 16) + 4 * lg + (k & 3);
        if constexpr (FP8) {
          const u32x2 c = *(const u32x2*)(st + L::at(r, 8 * w + (l16 >> 1)) + 8 * (l16 & 1));
          v[k] = codes_to_bf16(c[0], c[1]);
        } else {
          v[k] = *(const u32x4*)(st + L::at(r, 16 * w + l16));
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
        u32x4 av;
#pragma unroll
        for (int k = 0; k < 4; ++k) av[k] = __builtin_amdgcn_perm(v[2 * k + 1][c >> 1], v[2 * k][c >> 1], sel);
#pragma unroll
        for (int part = 1; part >= 0; --part)
          acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), p[part], acc[c], 0, 0, 0);
      }
    }
    lds_barrier();  // every wave is done with this stage and these products
    if (i + 2 < nblk) issue(i + 2);
  }
  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  if (w == 0 && it.rnew >= 0 && it.rnew < (a.max_pages << a.page_shift)) {
    const int64_t row = paged_row(a, slot, g, it.rnew);
    if (row >= 0) {
      unsigned char* to = (unsigned char*)const_cast<void*>(a.ck) + row * L::RB;
      if constexpr (FP8) {
        if (lane < L::CPR) {
          const u32x4* src = (const u32x4*)knew + 2 * lane;
          const u32x2 c0 = bf16_to_codes(src[0], ksc), c1 = bf16_to_codes(src[1], ksc);
          *(u32x4*)(to + 16 * lane) = u32x4{c0[0], c0[1], c1[0], c1[1]};
        }
      } else {
        for (int c = lane; c < L::CPR; c += 64) *(u32x4*)(to + 16 * c) = *((const u32x4*)knew + c);
      }
      if (lane == 0 && a.token) a.token[row] = a.pos[slot];
      if (lane == 0 && a.weight) a.weight[row] = 0.f;
    }
  }
  if (!hval) return;
  const size_t pi = (size_t)bid_x() * a.G + l16;
  if (w == 0 && lg == 0) a.ml[pi] = make_float2(m, lsum);
  float* dst = a.part + pi * DV + 128 * w + 8 * 4 * lg;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int c = 0; c < 8; c += 4)
      *(f32x4*)(dst + 8 * e + c) = f32x4{acc[c][e], acc[c + 1][e], acc[c + 2][e], acc[c + 3][e]} * ksc;
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
__global__ __launch_bounds__(kJoinThreads, 6) void paged_join(PagedArgs a, int merges) {
  constexpr int DG = DV / 4, CL = kJoinThreads / DG;
  __shared__ f32x4 sacc[kJoinThreads];
  __shared__ float2 sml[16];
  const int t = tid(), w = uniform(t >> 6);
  if (bid_x() < merges) {
    const int slices = a.dv / DV, sl = bid_x() % slices, bh = bid_x() / slices;
    const int b = bh / a.Hq, qh = bh % a.Hq, g = qh / a.G, h = qh % a.G;
    PagedSeq s;
    if (!paged_seq(a, b, false, s) || s.slot < 0 || s.slot >= a.n_slots) return;
    const int dg = t % DG, cl = t / DG;
    const size_t p0 = (size_t)(s.item0 + g * s.items) * a.G + h;
    const float* part = a.part + p0 * a.dv + sl * DV + 4 * dg;
    const size_t step = (size_t)a.G * a.dv;
    // the first kHeld partials of the thread are in flight with the references
    constexpr int kHeld = 8;
    f32x4 held[kHeld];
    float mheld[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = min(cl + j * CL, s.items - 1);
      if (s.items > 0) {
        held[j] = *(const f32x4*)(part + i * step);
        mheld[j] = a.ml[p0 + (size_t)i * a.G].x;
      }
    }
    const float2 ml = joined_ml(a, s, g, h);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    // an item none of whose rows is there has accumulated zeros
    auto add = [&](f32x4 v, float mi) { o += v * (mi == -INFINITY ? 0.f : fast_exp2(mi - ml.x)); };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (cl + j * CL < s.items) add(held[j], mheld[j]);
#pragma unroll 4
    for (int i = cl + kHeld * CL; i < s.items; i += CL) add(*(const f32x4*)(part + i * step), a.ml[p0 + (size_t)i * a.G].x);
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
  // two fours of rows (each of one page) a thread at a time, looked up ahead
  auto row_at = [&](int r) { return r < it.r1 ? paged_row(a, it.s.slot, it.g, r) : (int64_t)-1; };
  int r = it.r0 + 4 * t;
  int64_t row0 = row_at(r), row1 = row_at(r + 4 * kJoinThreads);
  for (int h = w; h < a.G; h += kJoinThreads / 64) {
    const float2 ml = joined_ml(a, it.s, it.g, h);
    if ((t & 63) == 0) sml[h] = make_float2(ml.x, ml.y > 0.f ? 1.f / ml.y : 0.f);
  }
  __syncthreads();
  const float* z = a.z + (it.s.block0 + (int64_t)it.g * it.s.blocks) * a.G * kBlockRows;
  while (r < it.r1) {
    const int q = r + 4 * kJoinThreads;
    const f32x4 v0 = new_weights(a, z, sml, row0, r, -1), v1 = new_weights(a, z, sml, row1, q, -1);
    put_weights(a, row0, r, it.r1, v0);
    put_weights(a, row1, q, it.r1, v1);
    r += 8 * kJoinThreads;
    row0 = row_at(r);
    row1 = row_at(r + 4 * kJoinThreads);
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

// block x: tokens 32x .. 32x + 31, y: KV head, z: sequence.  HBM bound: four prompts of
// 32k tokens or fewer out of the packed projection (622 MB) 137 us, 4.5 TB/s (a copy:
// 4.7).
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

// A packed batch by its map: tokens 32x .. 32x + 31, y: KV head.
struct PagedMapArgs {
  const void* k_new;
  const void* v_new;
  void* ck;
  void* cv;
  const float* k_scale;
  const float* v_scale;
  int32_t* token;
  float* weight;
  const int32_t* slot_ids;
  const int32_t* seq_of;
  const int32_t* row_of;
  const int32_t* pos_of;
  int64_t ks[2], vs[2];
  int64_t rows;  // of all pages, for one KV head
  int n, tokens, Hkv, dk, dv, n_slots, page_shift;
};
template <typename In, typename Out>
__global__ __launch_bounds__(256) void paged_append_mapped(PagedMapArgs a) {
  __shared__ int64_t rows[kAppendTokens];  // of this KV head among those of all pages, or -1
  __shared__ float scales[2][kAppendTokens];
  const int g = bid_y(), kc = a.dk / 8, vc = a.v_new ? a.dv / 8 : 0, t0 = bid_x() * kAppendTokens;
  if (tid() < kAppendTokens) {
    const int t = t0 + tid();
    const int r = t < a.tokens ? a.row_of[t] : -1, b = t < a.tokens ? a.seq_of[t] : -1;
    const int slot = b >= 0 && b < a.n ? a.slot_ids[b] : -1;
    int64_t row = -1;
    if (r >= 0 && r < a.rows && slot >= 0 && slot < a.n_slots) {
      row = (((int64_t)(r >> a.page_shift) * a.Hkv + g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
      if (sizeof(Out) == 1) {
        scales[0][tid()] = a.k_scale[(size_t)slot * a.Hkv + g];
        if (vc) scales[1][tid()] = a.v_scale[(size_t)slot * a.Hkv + g];
      }
      if (a.token) a.token[row] = a.pos_of[t];
      if (a.weight) a.weight[row] = 0.f;
    }
    rows[tid()] = row;
  }
  __syncthreads();
#pragma unroll 4
  for (int i = tid(); i < kAppendTokens * (kc + vc); i += 256) {
    const int at = i / (kc + vc), c = i % (kc + vc), t = t0 + at;
    const int64_t row = rows[at];
    if (row < 0) continue;
    if (c < kc)
      store8<In, Out>((const In*)a.k_new + t * a.ks[0] + g * a.ks[1] + 8 * c, (Out*)a.ck + row * a.dk + 8 * c,
                      sizeof(Out) == 1 ? scales[0][at] : 1.f);
    else
      store8<In, Out>((const In*)a.v_new + t * a.vs[0] + g * a.vs[1] + 8 * (c - kc), (Out*)a.cv + row * a.dv + 8 * (c - kc),
                      sizeof(Out) == 1 ? scales[1][at] : 1.f);
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

}  // namespace

SNAP_DEBUG_READER(debug_flags_paged)

// Work items that the card holds at once: more, shorter ones leave a partial
// second round, fewer leave loads unissued.  Latent rows: a workgroup a CU (fp8:
// two).  The others by the registers of a wave (two a SIMD): 2048, from 1024 items
// 224 -> 230 us on 128-wide fp32 rows, which fit one a SIMD, and 105 -> 102 (bf16)
// and 91 -> 59 (fp8) on 128-wide ones, 85 -> 56 on 64-wide bf16, all 32 x 4 heads of
// up to 16384 rows; from 3072 on all but 64-wide fp8 rows are slower (115, 61, 58).
// Those have half the bytes in flight a wave: 4096 items 46 -> 38 us, but with
// weights, whose staging leaves room for 2048, 59 -> 66.
static int resident_items(const snap_params& p, bool weigh) {
  if (p.d_qk == 576) return p.kv_dtype == SNAP_FP8_E4M3 ? 512 : 256;
  if (p.kv_dtype == SNAP_F32 && p.d_qk == 128) return 1024;
  return p.kv_dtype == SNAP_FP8_E4M3 && p.d_qk == 64 && !weigh ? 4096 : 2048;
}

// ---------------------------------------------------------------- host side
// The waves of a workgroup that takes a whole unit of 64- or 128-wide rows in one
// launch, or 0 where the rows are cut into items.  With few units one launch pays
// while a wave has four blocks of 64-wide rows, two of 128-wide ones or one of fp32
// (a further block is about 2 us of dependent work, the second launch 2.5); with
// enough units to fill the card, while it has eight, or four of 512 bytes a row and
// more (then also nothing is written for the join).  Measured, one launch / two, 32
// query heads on 8, us:
//   rows               256        512        1024       2048
//   128 bf16   1 x   8.9/11.5  10.8/11.5  15.3/11.3  23.9/11.3   64 x  21/24  30/35  48/55 100/95
//   128 fp8    1 x   8.7/11.1  10.7/11.3  14.4/11.2  21.2/11.6   64 x  17/21  25/27  34/36  53/56
//   64 fp8     1 x   8.5/11.1   8.5/11.1  11.2/11.2  16.5/11.3   64 x   9/20  12/22  19/28  28/40
//   64 fp32    1 x   8.6/11.2  12.1/11.3  18.1/11.3  29.3/11.2   64 x  20/26  30/36  49/56 102/97
//   128 fp32   1 x  12.6/11.3  18.7/11.3  29.2/11.4  50.1/12.4   64 x  31/37  50/58 106/103
// (two launches of one sequence are bound by the host; in a graph they take 9.4 to 12.3)
constexpr int kJoinedLogits = 6144;  // with weights: beside 32 KB for the join, within 64 KB of LDS
static int joined_waves(const snap_params& p, int n, int max_rows, bool weigh) {
  if (p.d_qk != p.d_v) return 0;
  const bool f32 = p.kv_dtype == SNAP_F32;
  const int blocks = (max_rows + kBlockRows - 1) / kBlockRows;
  const int waves = f32 && p.d_qk == 128 ? 4 : 8;  // by the registers of a wave
  const int row_bytes = (p.d_qk + p.d_v) * (f32 ? 4 : (p.kv_dtype == SNAP_BF16 ? 2 : 1));
  const int share = n * p.n_kv_heads * waves >= 2048 ? (row_bytes >= 512 ? 4 : 8) : (f32 ? 1 : (p.d_qk == 64 ? 4 : 2));
  const bool fits = !weigh || (int64_t)blocks * kBlockRows * (p.n_q_heads / p.n_kv_heads) <= kJoinedLogits;
  return blocks <= share * waves && fits ? waves : 0;
}

// Units that fill the card twice over and are short are an item each: the card
// balances them, and no workgroup reads every length to find its own.  What is lost is
// the cut of one long sequence among short ones, for which the bound on the rows
// stands.  Steps of 1000 (latent) and 520 (32 query heads on 8, 128-wide) bf16
// sequences, us, an item each / cut:
//   rows                    latent      128-wide
//   all 100                113 / 314    84 / 150
//   one of 2048, 2100      186 / 350   186 / 171
//   one of 4096            265 / 349   289 / 171
//   all 4096 (600, 520)    573 / 654  1460 / 1524
//   1 to 4096 (600, 520)   372 / 449   806 / 872
static bool whole_units(int units, int waves, int max_rows) { return units >= 2 * waves && max_rows <= 4096; }

PagedGeometry paged_geometry(const snap_params& p, int n, int max_rows, bool weigh) {
  PagedGeometry g{};
  const int units = (n > 0 ? n : 1) * p.n_kv_heads, G = p.n_q_heads / p.n_kv_heads;
  const int64_t blocks = (int64_t)units * ((max_rows + kBlockRows - 1) / kBlockRows);
  (PagedCut&)g = paged_cut(units, resident_items(p, weigh), blocks);
  size_t off = 0;
  g.off_part = off;
  off = align256(off + (size_t)g.max_items * G * p.d_v * sizeof(float));
  g.off_ml = off;
  off = align256(off + (size_t)g.max_items * G * sizeof(float2));
  g.off_z = off;
  if (weigh) {
    off = align256(off + (size_t)blocks * kBlockRows * G * sizeof(float));
    // (fewer items may be resident than without weights: room for those calls too)
    const size_t plain = paged_geometry(p, n, max_rows, false).bytes;
    if (off < plain) off = plain;
  }
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

snap_status launch_paged_append_mapped(const snap_params& p, const snap_paged_cache& c, int n, const int32_t* slot_ids,
                                       int tokens, const int32_t* seq_of, const int32_t* row_of, const int32_t* pos_of,
                                       const void* k_new, const int64_t* k_stride, const void* v_new,
                                       const int64_t* v_stride, hipStream_t stream) {
  PagedMapArgs a = {};
  a.k_new = k_new;
  a.v_new = p.v_in_k ? nullptr : v_new;
  a.ck = c.k;
  a.cv = p.v_in_k ? nullptr : c.v;
  a.k_scale = c.k_scale;
  a.v_scale = c.v_scale;
  a.token = c.token;
  a.weight = c.weight;
  a.slot_ids = slot_ids;
  a.seq_of = seq_of;
  a.row_of = row_of;
  a.pos_of = pos_of;
  a.rows = (int64_t)c.n_pages * c.page_size;
  a.n = n;
  a.tokens = tokens;
  a.Hkv = p.n_kv_heads;
  a.dk = p.d_qk;
  a.dv = p.d_v;
  a.n_slots = c.n_slots;
  a.page_shift = log2_of(c.page_size);
  const int64_t kd[2] = {(int64_t)p.n_kv_heads * p.d_qk, p.d_qk}, vd[2] = {(int64_t)p.n_kv_heads * p.d_v, p.d_v};
  for (int i = 0; i < 2; ++i) {
    a.ks[i] = k_stride ? k_stride[i] : kd[i];
    a.vs[i] = v_stride ? v_stride[i] : vd[i];
  }
  const dim3 grid((tokens + kAppendTokens - 1) / kAppendTokens, p.n_kv_heads);
  if (p.kv_dtype == SNAP_FP8_E4M3)
    hipLaunchKernelGGL((paged_append_mapped<uint16_t, uint8_t>), grid, dim3(256), 0, stream, a);
  else if (p.kv_dtype == SNAP_BF16)
    hipLaunchKernelGGL((paged_append_mapped<uint16_t, uint16_t>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_append_mapped<float, float>), grid, dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

snap_status launch_paged_decode(const snap_params& p, const snap_paged_cache& c, const int32_t* rows,
                                const int32_t* pos, int n, const int32_t* slot_ids, int max_rows, const void* q,
                                const void* k_new, const void* v_new, void* out, int out_dtype, bool weigh, void* ws,
                                hipStream_t stream) {
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
  a.waves = geo.waves;
  a.target = geo.target;
  a.max_items = geo.max_items;
  a.whole = whole_units(n * p.n_kv_heads, geo.waves, max_rows);
  a.out_bf16 = out_dtype == SNAP_BF16;
  split_scale2(p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_qk), a.scale2, a.scale2_lo);
  a.k_new = k_new;
  a.v_new = v_new;
  a.pos = pos;
  a.token = c.token;
  const size_t elt = p.kv_dtype == SNAP_F32 ? 4 : (p.kv_dtype == SNAP_BF16 ? 2 : 1);
  const size_t call_bytes = (size_t)n * p.n_kv_heads * max_rows * (p.d_qk + (p.v_in_k ? 0 : p.d_v)) * elt;
  const bool nt = p.kv_reuse == SNAP_KV_STREAM || (p.kv_reuse == SNAP_KV_AUTO && call_bytes >= kStreamingCallBytes);
  if (p.d_qk == 576) {
    static constexpr void (*kernels[2][2][2])(PagedArgs) = {  // [fp8][NT][W]
        {{paged_latent<false, false, false>, paged_latent<false, false, true>},
         {paged_latent<false, true, false>, paged_latent<false, true, true>}},
        {{paged_latent<true, false, false>, paged_latent<true, false, true>},
         {paged_latent<true, true, false>, paged_latent<true, true, true>}}};
    void (*k)(PagedArgs) = kernels[p.kv_dtype == SNAP_FP8_E4M3][nt][weigh];
    hipLaunchKernelGGL(k, dim3(geo.max_items), dim3(256), 0, stream, a);
  } else {
    const int kv = p.kv_dtype == SNAP_F32 ? kKvF32 : (p.kv_dtype == SNAP_BF16 ? kKvBf16 : kKvFp8);
    if (const int waves = joined_waves(p, n, max_rows, weigh)) {
      static constexpr void (*kernels[2][3][2])(PagedArgs) = {  // [width][type][W]
          {{paged_gqa<64, kKvBf16, false, false, 8>, paged_gqa<64, kKvBf16, false, true, 8>},
           {paged_gqa<64, kKvFp8, false, false, 8>, paged_gqa<64, kKvFp8, false, true, 8>},
           {paged_gqa<64, kKvF32, false, false, 8>, paged_gqa<64, kKvF32, false, true, 8>}},
          {{paged_gqa<128, kKvBf16, false, false, 8>, paged_gqa<128, kKvBf16, false, true, 8>},
           {paged_gqa<128, kKvFp8, false, false, 8>, paged_gqa<128, kKvFp8, false, true, 8>},
           {paged_gqa<128, kKvF32, false, false, 4>, paged_gqa<128, kKvF32, false, true, 4>}}};
      const int rows_pad = (max_rows + kBlockRows - 1) / kBlockRows * kBlockRows;
      hipLaunchKernelGGL(kernels[p.d_qk == 128][kv][weigh], dim3(n * p.n_kv_heads), dim3(64 * waves),
                         ((size_t)(waves / 2) * a.G * p.d_v + (weigh ? (size_t)rows_pad * a.G : 0)) * sizeof(float), stream, a);
      return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
    }
    static constexpr void (*kernels[2][3][2][2])(PagedArgs) = {  // [width][type][NT][W]
#define SNAP_PAGED_GQA(D, KV) \
  {{paged_gqa<D, KV, false, false, 1>, paged_gqa<D, KV, false, true, 1>}, {paged_gqa<D, KV, true, false, 1>, paged_gqa<D, KV, true, true, 1>}}
        {SNAP_PAGED_GQA(64, kKvBf16), SNAP_PAGED_GQA(64, kKvFp8), SNAP_PAGED_GQA(64, kKvF32)},
        {SNAP_PAGED_GQA(128, kKvBf16), SNAP_PAGED_GQA(128, kKvFp8), SNAP_PAGED_GQA(128, kKvF32)}};
#undef SNAP_PAGED_GQA
    void (*k)(PagedArgs) = kernels[p.d_qk == 128][kv][nt][weigh];
    hipLaunchKernelGGL(k, dim3(geo.max_items), dim3(64),
                       weigh ? (kZStage + kBlockRows * a.G) * sizeof(float) : 0, stream, a);
  }
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  // 128-dim slices (8 items at a time), or 32-dim ones (32 at a time) where a unit
  // has many items: 1 sequence x 8 KV heads of 32k rows, 256 items each, 9.4 -> 5.8 us
  const bool many = geo.max_items > 32 * n * p.n_kv_heads;
  const int merges = n * p.n_q_heads * (many ? p.d_v / 32 : (p.d_v == 512 ? 4 : 1));
  const dim3 join(merges + (weigh ? geo.max_items : 0));
  void (*j)(PagedArgs, int) = many ? paged_join<32> : (p.d_v == 64 ? paged_join<64> : paged_join<128>);
  hipLaunchKernelGGL(j, join, dim3(kJoinThreads), 0, stream, a, merges);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  return SNAP_OK;
}

}  // namespace snap
