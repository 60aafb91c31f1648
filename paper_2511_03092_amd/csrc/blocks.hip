// blocks.hip -- the block cache: rows in blocks of 32, 64 or 128 tokens, in 8 bits with
// a scale for each block and KV head, or in bf16, and attention of one new token over
// all of them or over those that a score selects.
//
//   block_append     a wave for each block of new keys or values
//   block_select     one workgroup for each (sequence, KV head), a unit: the blocks' scores
//                    from their bounds, and the best of them
//   block_score      the scores alone, where a unit's blocks are many
//   block_attn       one wave for each work item: a share of a unit's blocks, 32 rows of
//                    the newest token's own block, or that token stored
//   block_join       the items of a (sequence, query head) -> out
//   block_attn_unit  both for short calls, a workgroup a unit
#include <math.h>

#include "lds_dma.h"
#include "snap_internal.h"

namespace snap {

namespace {

enum { kRowsBf16 = 0, kRowsFp8 = 1, kRowsInt8 = 2 };

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

struct BlockArgs {
  const void* q;  // [n][Hq][d]
  unsigned char* ck;
  unsigned char* cv;
  float* ks;
  float* vs;
  unsigned char* kt;
  unsigned char* vt;
  int8_t* bound;
  float* bscale;
  const int32_t* rows;
  const int32_t* slot_ids;
  const int32_t* table;
  float* part;     // [items][G][d]  means of the items' values
  float2* ml;      // [items][G]  (max in log2 units, sum)
  int32_t* list;   // [units][list_ld] places of the selected blocks, ascending by block, then -1; NULL: all
  int32_t* sel_out;
  uint32_t* keys;  // [units][key_ld] the blocks' scores, where block_score forms them
  void* out;
  const void* k_new;  // a step's token, [n][Hkv][d]; NULL: the launch only attends
  const void* v_new;
  int n, Hq, Hkv, G, n_slots, n_pages, page_shift, block_shift, max_pages, max_rows, chosen, list_ld, key_ld, out_bf16;
  int waves, target, max_items;  // the cut (paged_cut.h)
  int sink, recent, best;  // selection: rows, rows, blocks
  float scale2, scale2_lo;
};

// One sequence of a call: the row of its newest token, its whole blocks before that
// one's, and whether that one's is attended.
struct BlockSeq {
  int slot, row, blocks;
  bool tail;
};
__device__ __forceinline__ BlockSeq block_seq(const BlockArgs& a, int b) {
  BlockSeq s;
  s.slot = a.slot_ids[b];
  const bool ok = s.slot >= 0 && s.slot < a.n_slots;
  s.row = ok ? a.rows[s.slot] : -1;
  s.row = uniform(s.row);
  s.slot = uniform(s.slot);
  if (!ok) s.row = -1;
  s.tail = s.row >= 0 && s.row < a.max_rows;
  s.blocks = s.row < 0 ? 0 : (s.tail ? s.row : a.max_rows) >> a.block_shift;
  return s;
}

// Index of a block of (slot, KV head g) among the blocks of all pages, or -1 when its
// page is not there.
__device__ __forceinline__ int block_at(const BlockArgs& a, int slot, int g, int block) {
  const int per = a.page_shift - a.block_shift, p = block >> per;
  if (p >= a.max_pages) return -1;
  const int page = a.table[(size_t)slot * a.max_pages + p];
  if (page < 0 || page >= a.n_pages) return -1;
  return (int)((((int64_t)page * a.Hkv + g) << per) + (block & ((1 << per) - 1)));
}

// Where the blocks of a call's units are cut: unit (b, g) has `items` work items from
// item0 + g items on.
struct BlockCut {
  int b, items, item0;
  int slot, blocks;  // (not where blocks are selected)
};

// The whole blocks of sequence b.
__device__ __forceinline__ int blocks_of(const BlockArgs& a, int b, int& slot) {
  slot = a.slot_ids[b];
  const bool ok = slot >= 0 && slot < a.n_slots;
  const int r = a.rows[ok ? slot : 0];  // no branch: the loads of several sequences go out together
  return !ok || r < 0 ? 0 : (r < a.max_rows ? r : a.max_rows) >> a.block_shift;
}

// Called by a whole wave.  by_item: the sequence that holds item `key`; otherwise
// sequence `key`.  false: there is none.
__device__ __forceinline__ bool block_cut(const BlockArgs& a, int key, bool by_item, BlockCut& c) {
  const int lane = tid() & 63;
  if (a.list) {  // selections are about as long as one another: the same items each
    c.items = a.max_items / (a.n * a.Hkv);
    c.b = by_item ? key / (c.items * a.Hkv) : key;
    c.item0 = c.b * a.Hkv * c.items;
    return c.b < a.n;
  }
  int64_t mine = 0;
  int nb0 = 0, slot0 = 0;
#pragma unroll 4
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    int slot;
    const int b = b0 + lane, blocks = blocks_of(a, min(b, a.n - 1), slot), nb = b < a.n ? blocks : 0;
    if (b0 == 0) {
      nb0 = nb;
      slot0 = slot;
    }
    mine += nb;
  }
  const int64_t total = wave_total((int)(mine & 0xfffff)) + ((int64_t)wave_total((int)(mine >> 20)) << 20);
  const int C = paged_chunk(a.waves, a.target, a.n, a.Hkv, total,
                            [&](int x) { return wave_total(x > 0 ? (nb0 + x - 1) / x : 0); });
  int before = 0;
  for (int b0 = 0; b0 < a.n; b0 += 64) {
    int slot = slot0, nb = nb0;
    const int b = b0 + lane;
    if (b0) {
      const int blocks = blocks_of(a, min(b, a.n - 1), slot);
      nb = b < a.n ? blocks : 0;
    }
    const int ni = (nb + C - 1) / C;
    const int si = wave_scan(ni), first = before + a.Hkv * (si - ni);
    const bool here = b < a.n && (by_item ? key >= first && key < first + a.Hkv * ni : key == b);
    const uint64_t m = __builtin_amdgcn_ballot_w64(here);
    if (m) {
      const int at = __builtin_ctzll(m);
      c.b = b0 + at;
      c.items = __builtin_amdgcn_readlane(ni, at);
      c.item0 = __builtin_amdgcn_readlane(first, at);
      c.slot = __builtin_amdgcn_readlane(slot, at);
      c.blocks = __builtin_amdgcn_readlane(nb, at);
      return debug_check(c.item0 + a.Hkv * c.items <= a.max_items, kDbgPagedItem);
    }
    before += a.Hkv * __builtin_amdgcn_readlane(si, 63);
  }
  return false;
}

// A loaded value is waited for here.  Before a loop, and behind a branch in one: where
// the compiler sees a load that may be in flight as the loop comes round, it waits at the
// value's use, every time, for all loads in flight.
template <typename T>
__device__ __forceinline__ void settle(T& v) {
  asm volatile("" : "+v"(v));
}

template <bool NT, typename T>
__device__ __forceinline__ T load_as(const void* p) {
  if constexpr (NT)
    return __builtin_nontemporal_load((const T*)p);
  else
    return *(const T*)p;
}

// ---------------------------------------------------------------- codes
constexpr float kLeastScale = 0x1p-126f;
__device__ __forceinline__ float block_scale(uint32_t amax_bf16, float top) {
  const float s = bf16_bits_to_f32(amax_bf16) * (1.f / top);
  return amax_bf16 == 0 ? 1.f : fmaxf(s, kLeastScale);
}

// Four values over a scale as int8 codes (NaN: 0, by its bits: the build lets float
// compares assume none).
__device__ __forceinline__ uint32_t int8x4(const float* x, float scale) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float y = fminf(fmaxf(__builtin_rintf(x[i] / scale), -127.f), 127.f);
    const uint32_t c = (__float_as_uint(x[i]) & 0x7fffffffu) > 0x7f800000u ? 0u : (uint32_t)(int)y & 0xffu;
    w |= c << (8 * i);
  }
  return w;
}

// 8 bf16 -> 8 codes
template <int KIND>
__device__ __forceinline__ u32x2 codes8(u32x4 raw, float scale) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_bits_to_f32(raw[i] & 0xffffu);
    f[2 * i + 1] = bf16_bits_to_f32(raw[i] >> 16);
  }
  if constexpr (KIND == kRowsInt8) {
    return u32x2{int8x4(f, scale), int8x4(f + 4, scale)};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] /= scale;
    return u32x2{e4m3x4_hw(f[0], f[1], f[2], f[3]), e4m3x4_hw(f[4], f[5], f[6], f[7])};
  }
}

// Largest finite magnitude of bf16 pieces, as bits.
__device__ __forceinline__ uint32_t amax8(u32x4 x, uint32_t m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
    m = max(m, lo < 0x7f80u ? lo : 0u);
    m = max(m, hi < 0x7f80u ? hi : 0u);
  }
  return m;
}
// Largest over rows of 16 lanes (to all of them) and over the wave, by lane shifts.
template <int CTRL>
__device__ __forceinline__ uint32_t turned(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __uint_as_float(turned<0x128>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(turned<0x124>(__float_as_uint(v))));
  v = fmaxf(v, __uint_as_float(turned<0x122>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(turned<0x121>(__float_as_uint(v))));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
  m = max(m, turned<0x128>(m));
  m = max(m, turned<0x124>(m));
  m = max(m, turned<0x122>(m));
  m = max(m, turned<0x121>(m));
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
             max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
}

// bf16 in an order of whole numbers (and back: its own inverse)
__device__ __forceinline__ int in_order(int h) { return (short)h < 0 ? (short)(h ^ 0x7fff) : (short)h; }
struct Bounds8 {
  int lo[8], hi[8];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = 0x7fff;
      hi[i] = -0x8000;
    }
  }
  __device__ __forceinline__ void add(u32x4 x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t h = (x[i >> 1] >> (16 * (i & 1))) & 0xffffu;
      const int k = in_order((int)h);
      const bool nan = (h & 0x7fffu) > 0x7f80u;
      lo[i] = nan ? lo[i] : min(lo[i], k);
      hi[i] = nan ? hi[i] : max(hi[i], k);
    }
  }
  __device__ __forceinline__ void join(int from) {  // with lane ^ from
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo[i] = min(lo[i], __shfl_xor(lo[i], from));
      hi[i] = max(hi[i], __shfl_xor(hi[i], from));
    }
  }
  // codes outwards, 8 bytes each
  __device__ __forceinline__ void codes(float scale, u32x2& least, u32x2& largest) const {
    least = largest = u32x2{0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool none = lo[i] > hi[i];
      const float l = bf16_bits_to_f32((uint32_t)in_order(lo[i]) & 0xffffu) / scale;
      const float h = bf16_bits_to_f32((uint32_t)in_order(hi[i]) & 0xffffu) / scale;
      const int cl = none ? 0 : (int)fminf(fmaxf(__builtin_floorf(l), -127.f), 127.f);
      const int ch = none ? 0 : (int)fminf(fmaxf(__builtin_ceilf(h), -127.f), 127.f);
      least[i >> 2] |= ((uint32_t)cl & 0xffu) << (8 * (i & 3));
      largest[i >> 2] |= ((uint32_t)ch & 0xffu) << (8 * (i & 3));
    }
  }
};

// A whole block's codes, scale and bounds written by one wave, from the rows that
// row(r) points to (bf16, read twice).  keys: it is the keys' side.
template <int D, int KIND, typename Row>
__device__ __forceinline__ void put_block(const BlockArgs& a, int at, bool keys, Row row) {
  constexpr int P = D / 8, R = 64 / P;  // pieces of a row, rows a wave takes at once
  const int lane = tid() & 63, col = lane % P, r0 = lane / P, B = 1 << a.block_shift;
  const bool bounds = keys && a.bound;
  if (KIND == kRowsBf16 && !bounds) return;
  uint32_t m = 0;
  Bounds8 bd;
  bd.init();
  constexpr int N = 4;  // pieces in flight (B is a multiple of N R)
  for (int r = r0; r < B; r += N * R) {
    u32x4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *((const u32x4*)row(r + i * R) + col);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m = amax8(x[i], m);
      if (bounds) bd.add(x[i]);
    }
  }
  m = wave_max(m);
  if constexpr (KIND != kRowsBf16) {
    const float s = block_scale(m, KIND == kRowsInt8 ? 127.f : 448.f);
    unsigned char* to = (keys ? a.ck : a.cv) + ((size_t)at << a.block_shift) * D + 8 * col;
    for (int r = r0; r < B; r += N * R) {
      u32x4 x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = *((const u32x4*)row(r + i * R) + col);
#pragma unroll
      for (int i = 0; i < N; ++i) *(u32x2*)(to + (size_t)(r + i * R) * D) = codes8<KIND>(x[i], s);
    }
    if (lane == 0) (keys ? a.ks : a.vs)[at] = s;
  }
  if (bounds) {
#pragma unroll
    for (int o = P; o < 64; o <<= 1) bd.join(o);
    const float s = block_scale(m, 127.f);
    u32x2 least, largest;
    bd.codes(s, least, largest);
    if (lane < P) {
      *(u32x2*)(a.bound + (size_t)at * 2 * D + 8 * col) = least;
      *(u32x2*)(a.bound + (size_t)at * 2 * D + D + 8 * col) = largest;
    }
    if (lane == 0) a.bscale[at] = s;
  }
}

// The same from registers, where every value is finite and of a middling size (else
// put_block does it): all rows are in flight at once and read once.
// Two bf16 a word: least and largest in whole numbers whose order is theirs, which give
// the largest magnitude too (a negative one of magnitude m is the number -1 - m).
// The quotient x / s of each code is off by 1.5 steps at most when it is x * fl(1 / s):
// an int8 code is rounded from that (by adding 1.5 * 2^23, whose last byte is then the
// code) unless it lies next to a tie, where the division is made; an E4M3 code from the
// quotient itself, which two corrections by the remainder give (a correctly rounded
// reciprocal and a quotient off by less than a step give it in one).
constexpr float kRoundMagic = 12582912.f;  // 1.5 * 2^23
template <int KIND>
__device__ __forceinline__ u32x2 quick_codes8(u32x4 raw, float scale, float inv) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(raw[i] << 16);
    f[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
  }
  if constexpr (KIND == kRowsInt8) {
    uint32_t c[8];
    float off = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float r = fmaf(f[i], inv, kRoundMagic);
      c[i] = __float_as_uint(r);
      off = fmaxf(off, fabsf(fmaf(f[i], inv, kRoundMagic - r)));
    }
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x0c0c0400u),
                                   __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x0c0c0400u), 0x05040100u);
    if (wave_any(off > 0.5f - 0x1p-15f)) {
      const u32x2 e = codes8<KIND>(raw, scale);
      if (off > 0.5f - 0x1p-15f) w = e;
    }
    return w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y = f[i] * inv;
      y = fmaf(fmaf(-scale, y, f[i]), inv, y);
      f[i] = fmaf(fmaf(-scale, y, f[i]), inv, y);
    }
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e4m3_v2i16 r = {0, 0};
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i], f[4 * i + 1], 1.0f, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i + 2], f[4 * i + 3], 1.0f, true);
      w[i] = __builtin_bit_cast(uint32_t, r);
    }
    return w;
  }
}

template <int D, int KIND, int B, typename Row>
__device__ __forceinline__ void put_block_at_once(const BlockArgs& a, int place, bool keys, Row row) {
  constexpr int P = D / 8, R = 64 / P, NP = B / R;
  const int lane = tid() & 63, col = lane % P, r0 = lane / P;
  const bool bounds = keys && a.bound;
  if (KIND == kRowsBf16 && !bounds) return;
  u32x4 x[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) x[p] = *((const u32x4*)row(p * R + r0) + col);
  const int at = uniform(place);  // (looked up while the rows are in flight)
  if (at < 0) return;
  i16x2 lo[4], hi[4], m = {0, 0};
  if (bounds) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t raw = x[p][i];  // (a vector's element as such would be cast as its first)
        const i16x2 h = __builtin_bit_cast(i16x2, raw), k = h ^ ((h >> 15) & (short)0x7fff);
        lo[i] = p ? __builtin_elementwise_min(lo[i], k) : k;
        hi[i] = p ? __builtin_elementwise_max(hi[i], k) : k;
      }
#pragma unroll
    for (int o = P; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_elementwise_min(lo[i], __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, lo[i]), o)));
        hi[i] = __builtin_elementwise_max(hi[i], __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, hi[i]), o)));
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_elementwise_max(hi[i], ~lo[i]));
  } else {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(i16x2, x[p][i] & 0x7fff7fffu));
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = __builtin_elementwise_max(m, __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, m), o)));
  const int amax = uniform(max((int)m[0], (int)m[1]));
  // magnitudes of 2^-60 to 2^60
  if (amax < (127 - 60) << 7 || amax >= (127 + 60) << 7) {
    put_block<D, KIND>(a, at, keys, row);
    return;
  }
  if constexpr (KIND != kRowsBf16) {
    const float s = block_scale(amax, KIND == kRowsInt8 ? 127.f : 448.f), inv = 1.f / s;
    unsigned char* to = (keys ? a.ck : a.cv) + ((size_t)at * B + r0) * D + 8 * col;
#pragma unroll
    for (int p = 0; p < NP; ++p) *(u32x2*)(to + p * R * D) = quick_codes8<KIND>(x[p], s, inv);
    if (lane == 0) (keys ? a.ks : a.vs)[at] = s;
  }
  if (bounds && lane < P) {
    const float s = block_scale(amax, 127.f);
    Bounds8 bd;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      bd.lo[i] = lo[i >> 1][i & 1];
      bd.hi[i] = hi[i >> 1][i & 1];
    }
    u32x2 least, largest;
    bd.codes(s, least, largest);
    *(u32x2*)(a.bound + (size_t)at * 2 * D + 8 * col) = least;
    *(u32x2*)(a.bound + (size_t)at * 2 * D + D + 8 * col) = largest;
    if (lane == 0) a.bscale[at] = s;
  }
}

// A step's token of a unit stored, keys or values: its row in the tail (bf16: the page),
// and the block's codes and bounds when it is the last of one.
template <int D, int KIND>
__device__ __forceinline__ void put_token(const BlockArgs& a, int unit, bool keys) {
  const int b = unit / a.Hkv, g = unit % a.Hkv, B = 1 << a.block_shift, lane = tid() & 63;
  const BlockSeq s = block_seq(a, b);
  if (s.row < 0) return;
  const int at = uniform(block_at(a, s.slot, g, s.row >> a.block_shift)), newest = s.row & (B - 1);
  if (at < 0) return;
  unsigned char* rows = KIND == kRowsBf16 ? (keys ? a.ck : a.cv) + ((size_t)at << a.block_shift) * D * 2
                                          : (keys ? a.kt : a.vt) + (((size_t)s.slot * a.Hkv + g) << a.block_shift) * D * 2;
  const unsigned char* in = (const unsigned char*)(keys ? a.k_new : a.v_new) + (size_t)unit * D * 2;
  if (lane < D / 8) *((u32x4*)(rows + newest * (D * 2)) + lane) = *((const u32x4*)in + lane);
  if (newest != B - 1) return;
  auto row = [&](int r) { return r == newest ? in : rows + r * (D * 2); };
  if (B == 32)
    put_block_at_once<D, KIND, 32>(a, at, keys, row);
  else if (B == 64)
    put_block_at_once<D, KIND, 64>(a, at, keys, row);
  else if (D == 64)
    put_block_at_once<64, KIND, 128>(a, at, keys, row);
  else  // (128 registers of rows would cost the attention a wave a SIMD)
    put_block<D, KIND>(a, at, keys, row);
}

// ---------------------------------------------------------------- append
struct BlockAppend {
  BlockArgs c;
  const int32_t* lengths;
  const int32_t* starts;
  int64_t ks[3], vs[3];  // bytes
  int tokens, max_len;
};

// Even waves take keys, odd ones values.  Workgroup 0: the sequence's first new block, and
// (8 bits, where that is not the last one) the last block's rows into the tail, stored
// after the barrier, behind which nobody reads the tail's old rows any more; workgroup x:
// blocks 2 x - 1 and 2 x.  HBM bound: four prompts of 32k tokens or fewer out of the packed
// projection into int8 (465 MB) 100 us, 4.6 TB/s (a copy: 4.7 to 4.9), without bounds 99;
// bf16 with bounds (618 MB) 137, without 129.  Short calls, 16 chunks of up to 512 64-wide
// rows into E4M3: 9.8 us, of which bounds 2.5 (joins over the lanes, then 16 divisions in
// D / 8 of them), scales and codes 1.1.
template <int D, int KIND, int B>
__global__ __launch_bounds__(256) void block_append(BlockAppend p) {
  const BlockArgs& a = p.c;
  constexpr int P = D / 8, R = 64 / P;
  const int w = uniform(tid() >> 6), lane = tid() & 63, col = lane % P, r0 = lane / P;
  const int g = bid_y(), b = __builtin_amdgcn_workgroup_id_z(), j = bid_x() ? 2 * bid_x() - 1 + (w >> 1) : 0;
  const bool keys = !(w & 1);
  // (loads that do not wait for one another go out together)
  int slot = a.slot_ids[b];
  int t0 = p.starts ? p.starts[b] : 0, len = p.starts ? p.starts[b + 1] : (p.lengths ? p.lengths[b] : p.max_len);
  const bool ok = slot >= 0 && slot < a.n_slots;
  const int row0 = uniform(a.rows[ok ? slot : 0]);
  slot = uniform(slot);
  if (!ok || row0 < 0) return;
  t0 = uniform(t0);
  len = uniform(len);
  if (p.starts) {
    t0 = min(max(t0, 0), p.tokens);
    len = min(max(len, 0), p.tokens) - t0;
  }
  len = min(len, p.max_len);
  const int64_t room = ((int64_t)a.max_pages << a.page_shift) - row0;
  if (len > room) len = room < 0 ? 0 : (int)room;
  if (len <= 0) return;
  const int first = row0 >> a.block_shift, skip = row0 & (B - 1), last = (skip + len - 1) >> a.block_shift;
  if (j > last) return;
  const int64_t* st = keys ? p.ks : p.vs;
  const unsigned char* in = (const unsigned char*)(keys ? a.k_new : a.v_new) + (p.starts ? 0 : b * st[0]) + g * st[1];
  unsigned char* tail = KIND == kRowsBf16 ? nullptr : (keys ? a.kt : a.vt) + ((((size_t)slot * a.Hkv + g) << a.block_shift) * D) * 2;
  auto given = [&](int i, int r) { return in + (t0 + (int64_t)i * B + r - skip) * st[2]; };
  // rows [from, upto) of block i, which come from the input, to their places behind `to`
  auto copy = [&](int i, unsigned char* to, int from, int upto, bool wait) {
    constexpr int NP = B / R;
    u32x4 x[NP];
#pragma unroll
    for (int q = 0; q < NP; ++q)
      if (q * R + r0 >= from && q * R + r0 < upto) x[q] = *((const u32x4*)given(i, q * R + r0) + col);
    if (wait) __syncthreads();
#pragma unroll
    for (int q = 0; q < NP; ++q)
      if (q * R + r0 >= from && q * R + r0 < upto) *((u32x4*)(to + (size_t)(q * R + r0) * D * 2) + col) = x[q];
  };
  const int upto = min(B, skip + len - j * B), from = j ? 0 : skip;
  const int at = block_at(a, slot, g, first + (bid_x() == 0 && w >= 2 ? last : j));
  if (bid_x() == 0 && w >= 2) {
    if (KIND != kRowsBf16 && last > 0) copy(last, tail, 0, uniform(at) < 0 ? 0 : skip + len - last * B, true);
    return;
  }
  unsigned char* old = KIND == kRowsBf16 ? (keys ? a.ck : a.cv) + ((size_t)max(at, 0) << a.block_shift) * D * 2 : tail;
  if (upto == B)
    put_block_at_once<D, KIND, B>(a, at, keys, [&](int r) -> const unsigned char* { return r < from ? old + (size_t)r * D * 2 : given(j, r); });
  if (KIND == kRowsBf16 || last == 0) {
    if (uniform(at) >= 0) copy(j, old, from, upto, false);
  } else if (bid_x() == 0) {
    __syncthreads();
  }
}

// ---------------------------------------------------------------- selection
constexpr int kSelThreadsB = 1024, kSelWaves = kSelThreadsB / 64;
constexpr uint32_t kForced = 0xffffffffu;  // above every score's key; 0, below them: no such block

// A score's bits in the order of whole numbers, within [1, kForced - 1].
__device__ __forceinline__ uint32_t score_key(float s) {
  const uint32_t u = __float_as_uint(s + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Largest bin of a falling search: the bin of hist[0 .. 1023] that holds the rem-th
// largest, how many are in the bins above it and in it; {-1, ..} when there are fewer.
// Called by one wave.
__device__ __forceinline__ void find_bin(const int* hist, int rem, int* out) {
  const int lane = tid() & 63;
  int c[16], sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const i32x4 v = *(const i32x4*)(hist + 1008 - 16 * lane + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += c[4 * i + e] = v[e];
  }
  const int upto = wave_scan(sum);
  int before = upto - sum;
  if (lane == 63 && upto < rem) out[0] = -1;
  if (before < rem && rem <= upto) {
    int bin = 0, above = before, in = 0;
#pragma unroll
    for (int i = 15; i >= 0; --i) {
      if (before < rem && rem <= before + c[i]) {
        bin = 1008 - 16 * lane + i;
        above = before;
        in = c[i];
      }
      before += c[i];
    }
    out[0] = bin;
    out[1] = above;
    out[2] = in;
  }
}

// What a unit's selection goes by: blocks [0, f0) and [f1, nb) are selected whatever
// their scores; those between are scored where there are more than `best` of them.
struct BlockChoice {
  const int32_t* table;  // the slot's pages
  int g, per, nb, f0, f1;
  bool scored;
  __device__ __forceinline__ int page(const BlockArgs& a, int j) const { return table[min(j >> per, a.max_pages - 1)]; }
  // index of block j among the blocks of all pages, from its page; -1: not there
  __device__ __forceinline__ int place(const BlockArgs& a, int j, int page) const {
    return page < 0 || page >= a.n_pages ? -1 : (int)((((int64_t)page * a.Hkv + g) << per) + (j & ((1 << per) - 1)));
  }
  __device__ __forceinline__ bool there(const BlockArgs& a, int j) const { return place(a, j, page(a, j)) >= 0; }
};
// The slot's pages first; its rows (whose loads wait for the slot's id as well) by limits().
__device__ __forceinline__ BlockChoice choice_of(const BlockArgs& a, int unit, int& held) {
  BlockChoice c;
  c.g = unit % a.Hkv;
  c.per = a.page_shift - a.block_shift;
  const int slot = a.slot_ids[unit / a.Hkv];
  const bool ok = slot >= 0 && slot < a.n_slots;
  c.table = a.table + (size_t)(ok ? slot : 0) * a.max_pages;
  held = a.rows[ok ? slot : 0];
  held = ok ? held : -1;
  c.f0 = (int)(((int64_t)a.sink + (1 << a.block_shift) - 1) >> a.block_shift);
  return c;
}
__device__ __forceinline__ void limits(const BlockArgs& a, int held, BlockChoice& c) {
  const int row = uniform(held);
  c.nb = row < 0 ? 0 : min(row, a.max_rows) >> a.block_shift;
  c.f0 = min(c.nb, c.f0);
  const int f1 = row - (a.recent - 1);
  c.f1 = max(c.f0, min(c.nb, f1 <= 0 ? 0 : f1 >> a.block_shift));
  c.scored = c.f1 - c.f0 > a.best && a.best > 0;
}

// The keys of blocks [first, end) of a unit, by a workgroup of W waves: wave w scores 16
// blocks at a time, N times 16 of them in flight.  The scores are products of 8-bit whole
// numbers on the matrix units, exact in 32 bits, so that a choice does not depend on the
// order of sums.  qraw: wave w's share of the queries, [(G + W - 1) / W]; pages: those of
// the wave's first blocks.
template <int D, int W>
struct BlockScores {
  static constexpr int NK = 2 * D / 64, N = (D == 128 ? 2 : 4) * (W == kSelWaves ? 1 : 2), kStep = 16 * W, Q = 16 / W;
  static constexpr int kBatch = kStep * N;  // blocks in flight
  static constexpr int P = 2 * D / 16;  // 16-byte pieces of a block's bounds
  struct Shared {
    int8_t a[16][2 * D];  // a query's codes: those below zero, then those above
    float u[16];
    u32x4 x[W][16 * P];  // a wave's 16 blocks
  };
  // Where piece p of block r of 16 stands: turned, so that neither the rows that are
  // written nor the columns that are read meet on a bank.
  static __device__ __forceinline__ int spot(int r, int p) { return r * P + (p ^ (P == 16 ? r : (r >> 1) & 7)); }
  int pages[N];
  uint32_t qraw[Q][D / 64];
  __device__ __forceinline__ void load_q(const BlockArgs& a, int unit) {
    const int w = tid() >> 6, lane = tid() & 63, b = unit / a.Hkv, g = unit % a.Hkv;
#pragma unroll
    for (int k = 0; k < Q; ++k)
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        qraw[k][i] = ((const uint16_t*)a.q)[((size_t)b * a.Hq + g * a.G + min(w + W * k, a.G - 1)) * D + i * 64 + lane];
  }
  __device__ __forceinline__ void load_pages(const BlockArgs& a, const BlockChoice& c, int j) {
#pragma unroll
    for (int i = 0; i < N; ++i) pages[i] = c.page(a, j + kStep * i + (tid() & 15));
  }
  template <typename Emit>
  __device__ __forceinline__ void run(const BlockArgs& a, const BlockChoice& c, int first, int end, Shared& sh, Emit emit) {
    const int lane = tid() & 63, w = uniform(tid() >> 6), l16 = lane & 15, lg = lane >> 4;
    int at[N];
    float bs[N];
    // Loads take 1 KB of neighbouring bytes (with the rows of a matrix operand a lane each,
    // 64 bytes of 16 blocks, the L1 passes 16 bytes a clock); the operand is made in LDS.
    u32x4 x[N][NK];
    // blocks j1 + l16 into place i, and the page of those that follow there
    auto load = [&](int i, int j1) {
      if (j1 >= end) return;  // (the whole wave)
      const int j = j1 + l16;
      at[i] = j < end ? c.place(a, j, pages[i]) : -1;
      bs[i] = a.bscale[max(at[i], 0)];
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const int piece = 64 * k + lane, block = __shfl(at[i], piece / P);
        x[i][k] = *(const u32x4*)(a.bound + ((size_t)max(block, 0) * P + piece % P) * 16);
      }
      if (j1 + kBatch < end) pages[i] = c.page(a, j + kBatch);
    };
    int j0 = first + 16 * w;
#pragma unroll
    for (int i = 0; i < N; ++i) load(i, j0 + kStep * i);
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const int h = w + W * k;
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint32_t mag = h < a.G ? qraw[k][i] & 0x7fffu : 0u;
        m = max(m, mag < 0x7f80u ? mag : 0u);
      }
      const float u = block_scale(wave_max(m), 127.f);
      if (lane == 0) sh.u[h] = u;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint32_t v = h < a.G ? qraw[k][i] : 0u;
        const float y = fminf(fmaxf(__builtin_rintf(bf16_bits_to_f32(v) / u), -127.f), 127.f);
        const int z = (v & 0x7fffu) > 0x7f80u ? 0 : (int)y;  // (NaN)
        sh.a[h][i * 64 + lane] = (int8_t)min(z, 0);
        sh.a[h][D + i * 64 + lane] = (int8_t)max(z, 0);
      }
    }
    lds_barrier();  // (the blocks' loads stay in flight)
    i32x4 q[NK];
#pragma unroll
    for (int i = 0; i < NK; ++i) q[i] = *(const i32x4*)(&sh.a[l16][64 * i + 16 * lg]);
    const float u = sh.u[l16];
    for (; j0 < end; j0 += kBatch) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int j1 = j0 + kStep * i;
        if (j1 >= end) continue;
        i32x4 s = {0, 0, 0, 0};
        // (one wave's LDS operations take effect in order)
#pragma unroll
        for (int k = 0; k < NK; ++k) sh.x[w][spot((64 * k + lane) / P, (64 * k + lane) % P)] = x[i][k];
        asm volatile("" ::: "memory");
#pragma unroll
        for (int k = 0; k < NK; ++k)
          s = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, sh.x[w][spot(l16, 4 * k + lg)]), q[k], s, 0, 0, 0);
        asm volatile("" ::: "memory");
        float best[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) best[e] = row_max(l16 < a.G ? (float)s[e] * u : -INFINITY);
        // lane (l16 < 4, lg) keeps block 4 lg + l16's; its scale and place are lane 4 lg + l16's
        const int from_lane = 4 * lg + (l16 & 3);
        const float mine = l16 == 0 ? best[0] : (l16 == 1 ? best[1] : (l16 == 2 ? best[2] : best[3]));
        const float scale = __shfl(bs[i], from_lane);
        const int place = __shfl(at[i], from_lane);
        if (l16 < 4 && j1 + from_lane < end) emit(j1 + from_lane, place < 0 ? 0u : score_key(mine * scale));
        load(i, j1 + kBatch);
      }
    }
  }
};

// The keys of a unit's blocks, cut over several workgroups where they are many.
constexpr int kScoreThreads = 256;
template <int D>
__global__ __launch_bounds__(kScoreThreads) void block_score(BlockArgs a) {
  typedef BlockScores<D, kScoreThreads / 64> Scores;
  constexpr int chunk = Scores::kBatch;
  __shared__ __align__(16) typename Scores::Shared sh;
  const int unit = bid_y();
  Scores s;
  s.load_q(a, unit);
  int held;
  BlockChoice c = choice_of(a, unit, held);
  const int first = c.f0 + bid_x() * chunk;
  s.load_pages(a, c, first + 16 * (tid() >> 6));
  limits(a, held, c);
  const int end = min(c.f1, first + chunk);
  if (!c.scored || first >= end) return;
  uint32_t* keys = a.keys + (size_t)unit * a.key_ld;
  s.run(a, c, first, end, sh, [&](int j, uint32_t k) { keys[j] = k; });
}

// One workgroup a unit, bound by dependent steps: 8 units of 512 blocks 11.5 us (queries,
// pages and bounds 5.5, the histograms 1.5, the list 1), 128 units of 2048 blocks 23 us, then
// mostly the bounds' 67 MB by 128 of 256 CUs.  The keys are in LDS.  The last score taken is found by a
// histogram over the range that the scores span, then over the bin that holds it, and so
// on until a bin is taken whole or is one score: two turns, mostly.  GIVEN: the keys are
// block_score's.
template <int D, bool GIVEN>
__global__ __launch_bounds__(kSelThreadsB) void block_select(BlockArgs a) {
  extern __shared__ __align__(16) uint32_t key[];  // one a block
  typedef BlockScores<D, kSelWaves> Scores;
  __shared__ __align__(16) typename Scores::Shared sh;
  __shared__ __align__(16) int hist[2][1024];
  __shared__ uint32_t range[kSelWaves][2];
  __shared__ int cnt[kSelWaves][2], out[3];
  const int t = tid(), lane = t & 63, w = uniform(t >> 6), unit = bid_x();
  Scores s;
  if constexpr (!GIVEN) s.load_q(a, unit);
  int held;
  BlockChoice c = choice_of(a, unit, held);
  if constexpr (!GIVEN) s.load_pages(a, c, c.f0 + 16 * w);
  hist[0][t] = 0;
  limits(a, held, c);
  const int nb = c.nb, f0 = c.f0, f1 = c.f1;
  // in flight with the bounds: the pages of the thread's forced block and of the first one
  // that it may write (wave w writes its share of the blocks, in order)
  const int share = ((nb + kSelWaves - 1) / kSelWaves + 63) & ~63, a0 = min(nb, w * share), a1 = min(nb, a0 + share);
  auto forced = [&](int i) { return i < f0 ? i : f1 + i - f0; };
  const int forced_page = c.page(a, forced(t)), own_page = c.page(a, a0 + lane);
  int32_t* list = a.list + (size_t)unit * a.list_ld;
  int32_t* sel = a.sel_out ? a.sel_out + (size_t)unit * a.chosen : nullptr;
  uint32_t T = 0;  // taken: above T, and the first `rem` of T
  int rem = a.best;
  uint32_t least = kForced, most = 0;
  auto keep = [&](int j, uint32_t k) {
    key[j] = k;
    if (k) {
      least = min(least, k);
      most = max(most, k);
    }
  };
  if (!c.scored) {
    for (int j = f0 + t; j < f1; j += kSelThreadsB) key[j] = a.best > 0 && c.there(a, j) ? kForced : 0u;
  } else if constexpr (GIVEN) {
    const uint32_t* keys = a.keys + (size_t)unit * a.key_ld;
#pragma unroll 4
    for (int j = f0 + t; j < f1; j += kSelThreadsB) keep(j, keys[j]);
  } else {
    s.run(a, c, f0, f1, sh, keep);
  }
  for (int i = t; i < f0 + nb - f1; i += kSelThreadsB) {
    const int j = forced(i);
    key[j] = c.place(a, j, i == t ? forced_page : c.page(a, j)) >= 0 ? kForced : 0u;
  }
  if (c.scored) {
    least = ~wave_max(~least);
    most = wave_max(most);
    if (lane == 0) {
      range[w][0] = least;
      range[w][1] = most;
    }
  }
  __syncthreads();
  if (c.scored) {
    uint32_t lo = kForced, hi = 0;
#pragma unroll
    for (int i = 0; i < kSelWaves; ++i) {
      lo = min(lo, range[i][0]);
      hi = max(hi, range[i][1]);
    }
    for (int turn = 0;; ++turn) {
      if (lo > hi) break;  // no block is there: nothing is above T that is not forced
      const int span = 32 - __builtin_clz((hi - lo) | 1u), shift = span > 10 ? span - 10 : 0;
      int* h = hist[turn & 1];
      for (int j = f0 + t; j < f1; j += kSelThreadsB) {
        const uint32_t k = key[j];
        if (k >= lo && k <= hi) atomicAdd(&h[(k - lo) >> shift], 1);
      }
      hist[~turn & 1][t] = 0;
      __syncthreads();
      if (w == 0) find_bin(h, rem, out);
      __syncthreads();
      const int bin = out[0];
      if (bin < 0) break;  // fewer than wanted are there at all: all of them are taken (T = 0)
      rem -= out[1];
      lo += (uint32_t)bin << shift;
      if (rem == out[2]) {  // all of the bin
        T = lo - 1;
        rem = 0;
        break;
      }
      if (shift == 0) {
        T = lo;
        break;
      }
      const uint32_t top = lo + ((1u << shift) - 1u);
      hi = top < hi ? top : hi;
      __syncthreads();  // (out is read before it is written again)
    }
  }
  int above = 0, equal = 0;
  for (int j = a0 + lane; j - lane < a1; j += 64) {
    const uint32_t k = j < a1 ? key[j] : 0u;
    above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k > T));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k != 0 && k == T));
  }
  if (lane == 0) {
    cnt[w][0] = above;
    cnt[w][1] = equal;
  }
  __syncthreads();
  int above0 = 0, equal0 = 0, aboves = 0, equals = 0;
#pragma unroll
  for (int i = 0; i < kSelWaves; ++i) {
    if (i < w) {
      above0 += cnt[i][0];
      equal0 += cnt[i][1];
    }
    aboves += cnt[i][0];
    equals += cnt[i][1];
  }
  const int total = aboves + min(equals, rem);
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int j = a0 + lane; j - lane < a1; j += 64) {
    const uint32_t k = j < a1 ? key[j] : 0u;
    const uint64_t am = __builtin_amdgcn_ballot_w64(k > T), em = __builtin_amdgcn_ballot_w64(k != 0 && k == T);
    const int e = equal0 + __builtin_popcountll(em & below), i = above0 + __builtin_popcountll(am & below) + min(e, rem);
    const bool take = k > T || (k != 0 && k == T && e < rem);
    if (take && debug_check(i < a.list_ld, kDbgBlockList) && i < a.list_ld) {
      list[i] = c.place(a, j, j == a0 + lane ? own_page : c.page(a, j));
      if (sel) sel[i] = j;
    }
    above0 += __builtin_popcountll(am);
    equal0 += __builtin_popcountll(em);
  }
  for (int i = total + t; i < a.list_ld; i += kSelThreadsB) list[i] = -1;
  if (sel)
    for (int i = total + t; i < a.chosen; i += kSelThreadsB) sel[i] = -1;
}

// ---------------------------------------------------------------- attention
constexpr float kStaleMax = 8.f;

// Eight weights as three bf16 terms, whose sum they are (pe is used up).  INF, for values
// that may be infinite: the second and third are kept off zero, so that an infinite value
// times them stays infinite, by 2^-32 of the weight itself (a floor that is the same for
// every weight would give large finite values a share that they do not have).
template <bool INF>
__device__ __forceinline__ void three_terms(float (&pe)[8], bf16x8 (&p)[3]) {
  float least[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) least[i] = INF ? pe[i] * 0x1p-32f : 0.f;
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    u32x4 pw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = INF && part ? fmaxf(pe[2 * i], least[2 * i]) : pe[2 * i];
      const float hi = INF && part ? fmaxf(pe[2 * i + 1], least[2 * i + 1]) : pe[2 * i + 1];
      pe[2 * i] -= __uint_as_float(__float_as_uint(pe[2 * i]) & 0xffff0000u);
      pe[2 * i + 1] -= __uint_as_float(__float_as_uint(pe[2 * i + 1]) & 0xffff0000u);
      pw[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
    p[part] = __builtin_bit_cast(bf16x8, pw);
  }
}

// 4 codes -> 4 bf16 (exact)
template <int KIND>
__device__ __forceinline__ u32x2 bf16x4(uint32_t c) {
  if constexpr (KIND == kRowsFp8) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, true))};
  } else {
    uint32_t f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __float_as_uint((float)(int)(int8_t)(c >> (8 * i)));
    return u32x2{__builtin_amdgcn_perm(f[1], f[0], 0x07060302u), __builtin_amdgcn_perm(f[3], f[2], 0x07060302u)};
  }
}

// The softmax of a query head (column l16) and its sum of values.  acc is in units of
// 2^unit, a power that each column has of its own, so that weights reach the matrix units
// in the middle of their range and acc stays finite where the mean of the values is:
//   codes: a weight is probability times scale; the unit is that of the largest product so
//     far (to within 2^8), whatever the size of the scales, and follows the reference as
//     that rises.  What is lost is below 2^-126 of the largest product.
//   rows as they came: a weight is a probability; the unit is at least the sum of them, so
//     that acc is at most the largest value, and 2^5 or that of the sum (to within 2^4).
//     What is lost is below 2^-121 of the sum.
constexpr int kRowsUnit = 5;        // 32 rows of a probability of at most 1
constexpr float kLeastRise = -110.f;  // so that scale / 2^unit is finite where the probabilities are next to nothing
template <int D>
struct Soft {
  static constexpr int VE = D / 16;  // value dims a lane
  float m = -INFINITY, mref = 0.f, lsum = 0.f, unit = kRowsUnit;
  f32x4 acc[VE];
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int c = 0; c < VE; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ float total() const {  // of lsum, over the lanes of a column
    const float s = lsum + __shfl_xor(lsum, 16);
    return s + __shfl_xor(s, 32);
  }
  // acc in the unit that rows as they came go by, from whatever it is in.
  __device__ __forceinline__ void by_total() {
    const int e = (int)(__float_as_uint(total()) >> 23) - 127;
    const float now = (float)(max(e, 0) + 4);
#pragma unroll
    for (int c = 0; c < VE; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[c][i] = __builtin_ldexpf(acc[c][i], (int)(unit - now));
    unit = now;
  }
  // Products x of eight rows at xs a unit (xlo: its low part) -> weights: probabilities times
  // scale (CODES), in units of 2^unit.
  template <bool CODES>
  __device__ __forceinline__ void softmax(const float (&x)[8], float xs, float xlo, float scale, float (&pe)[8]) {
    float bm = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    bm = fmaxf(bm, __shfl_xor(bm, 16));
    bm = fmaxf(bm, __shfl_xor(bm, 32));
    bm *= xs;
    const float es = (float)((int)(__float_as_uint(scale) >> 23) - 127);
    const bool up = bm > m + kStaleMax, far = CODES && fmaxf(bm - mref, kLeastRise) + es > unit + kStaleMax;
    if (wave_any(up || far)) {
      const float mnew = up ? bm : m, rise = up ? mnew - m : 0.f;  // (infinite at the first rows)
      m = mnew;
      mref = m == -INFINITY ? 0.f : m;
      const float least = CODES ? es + fmaxf(__builtin_ceilf(bm - mref), kLeastRise) : (float)kRowsUnit;
      const float alpha = fast_exp2(-rise), now = fmaxf(unit - __builtin_floorf(rise), least);
      const float beta = __builtin_ldexpf(alpha, (int)(unit - now));
#pragma unroll
      for (int c = 0; c < VE; ++c) acc[c] *= beta;
      lsum *= alpha;
      unit = now;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) pe[i] = fast_exp2(fmaf(x[i], xs, fmaf(x[i], xlo, -mref)));
    lsum += ((pe[0] + pe[1]) + (pe[2] + pe[3])) + ((pe[4] + pe[5]) + (pe[6] + pe[7]));
    // (a quarter of the unit in each of a column's four lanes)
    if (!CODES && wave_any(lsum > __builtin_ldexpf(0.25f, (int)unit))) by_total();
    const float w = __builtin_ldexpf(CODES ? scale : 1.f, -(int)unit);
#pragma unroll
    for (int i = 0; i < 8; ++i) pe[i] *= w;
  }
  // acc times f, in units of 1.  (CODES: by a middling power of two first, so that what is
  // between stays in range)
  template <bool CODES>
  __device__ __forceinline__ void by(float f) {
    const float h = CODES ? fminf(fmaxf(unit, -40.f), 40.f) : unit, g = __builtin_ldexpf(f, (int)h);
#pragma unroll
    for (int c = 0; c < VE; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[c][i] = CODES ? __builtin_ldexpf(acc[c][i] * g, (int)(unit - h)) : acc[c][i] * g;
  }
  // their sum over the rows' values, int8 codes: made bf16 in the operand's order
  template <typename Raw>
  __device__ __forceinline__ void values8(float (&pe)[8], const Raw (&v)[8]) {
    bf16x8 p[3];
    three_terms<false>(pe, p);
#pragma unroll
    for (int c = 0; c < VE; ++c) {
      u32x4 av;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = (float)(int)(int8_t)(v[2 * i][c >> 2] >> (8 * (c & 3)));
        const float y = (float)(int)(int8_t)(v[2 * i + 1][c >> 2] >> (8 * (c & 3)));
        av[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
      }
#pragma unroll
      for (int part = 2; part >= 0; --part)
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), p[part], acc[c], 0, 0, 0);
    }
  }
  // their sum over the rows' values (two bf16 a word)
  template <bool INF>
  __device__ __forceinline__ void values(float (&pe)[8], const uint32_t (&vw)[8][VE / 2]) {
    bf16x8 p[3];
    three_terms<INF>(pe, p);
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
};

// Rows r0 .. r0 + 31 of the newest token's block, as they came; the token itself is read
// from a step's input.
template <int D, int KIND>
__device__ __forceinline__ void attend_newest(const BlockArgs& a, const BlockSeq& s, int b, int g, int at, int r0, Soft<D>& o) {
  constexpr int VE = D / 16;
  typedef uint32_t VTail __attribute__((ext_vector_type(VE * 2 / 4)));
  const int lane = tid() & 63, l16 = lane & 15, lg = lane >> 4, B = 1 << a.block_shift, newest = s.row & (B - 1);
  const bool hval = l16 < a.G;
  const unsigned char* qp = (const unsigned char*)a.q + ((size_t)b * a.Hq + g * a.G + (hval ? l16 : 0)) * D * 2;
  const size_t t0 = (((size_t)s.slot * a.Hkv + g) << a.block_shift) * D * 2, p0 = ((size_t)at << a.block_shift) * D * 2;
  const unsigned char* kb = KIND == kRowsBf16 ? a.ck + p0 : a.kt + t0;
  const unsigned char* vb = KIND == kRowsBf16 ? a.cv + p0 : a.vt + t0;
  const size_t n0 = ((size_t)b * a.Hkv + g) * D * 2;
  const unsigned char* kn = a.k_new ? (const unsigned char*)a.k_new + n0 : kb + newest * (D * 2);
  const unsigned char* vn = a.k_new ? (const unsigned char*)a.v_new + n0 : vb + newest * (D * 2);
  const int ra = r0 + l16, rb = ra + 16;
  const unsigned char* pa = ra >= newest ? kn : kb + ra * (D * 2);  // (rows past the newest are masked)
  const unsigned char* pb = rb >= newest ? kn : kb + rb * (D * 2);
  u32x4 q[D / 32], k0[D / 32], k1[D / 32];
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    q[j] = hval ? *(const u32x4*)(qp + 64 * j + 16 * lg) : u32x4{0u, 0u, 0u, 0u};
    k0[j] = *(const u32x4*)(pa + 64 * j + 16 * lg);
    k1[j] = *(const u32x4*)(pb + 64 * j + 16 * lg);
  }
  VTail v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + (i < 4 ? 0 : 16) + 4 * lg + (i & 3);
    v[i] = *(const VTail*)((r >= newest ? vn : vb + r * (D * 2)) + l16 * (VE * 2));
  }
  f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k0[j]), __builtin_bit_cast(bf16x8, q[j]), s0, 0, 0, 0);
    s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k1[j]), __builtin_bit_cast(bf16x8, q[j]), s1, 0, 0, 0);
  }
  float x[8], pe[8];
  uint32_t vw[8][VE / 2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + (i < 4 ? 0 : 16) + 4 * lg + (i & 3);
    x[i] = r <= newest ? (i < 4 ? s0[i & 3] : s1[i & 3]) : -INFINITY;
    if (r > newest) v[i] = VTail{};
#pragma unroll
    for (int u = 0; u < VE / 2; ++u) vw[i][u] = v[i][u];
  }
  o.template softmax<false>(x, a.scale2, a.scale2_lo, 1.f, pe);
  o.template values<true>(pe, vw);
}

// The 32-row steps [first, end) of a unit's blocks (those listed, or all), by one wave for
// the G query heads of its KV head at once: products of 32 keys with the heads (padded to
// 16 columns) on the matrix units, an online softmax in the exp2 domain, the probabilities
// times a block's value scale, times the codes on the matrix units.  Lane (l16, lg) holds
// head l16's logits of rows 4 lg + e of each 16-row half, which is also what the second
// product takes from it; its keys are 16 bytes at byte 64 j + 16 lg of row l16, its values
// the D / 16 dims from (D / 16) l16 of eight rows.  Every row of a whole block is there, so
// nothing is masked.  HBM bound: 8 sequences of 4k to 128k int8 rows x 8 KV heads (1.26 GB)
// 203 us, 6.2 TB/s with the join; 32 of up to 16k E4M3 rows (554 MB) 100 us.
// AHEAD: the values are loaded a step before they are needed, as the keys are; that changes
// nothing where the card is full of waves.
template <int D, int KIND, bool NT, bool AHEAD>
__device__ __forceinline__ void attend_blocks(const BlockArgs& a, int b, int g, int slot, const int32_t* list, int first, int end, Soft<D>& o) {
  constexpr int E = KIND == kRowsBf16 ? 2 : 1, VE = D / 16, NK = D * E / 64;
  typedef uint32_t VRaw __attribute__((ext_vector_type(VE * E / 4)));
  const int lane = tid() & 63, l16 = lane & 15, lg = lane >> 4, B = 1 << a.block_shift, steps = a.block_shift - 5;
  const bool hval = l16 < a.G;
  const unsigned char* qp = (const unsigned char*)a.q + ((size_t)b * a.Hq + g * a.G + (hval ? l16 : 0)) * D * 2;
  u32x4 q[D / 32];
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    const int off = KIND == kRowsBf16 ? 64 * j + 16 * lg : (64 * (j / 2) + 16 * lg + 8 * (j & 1)) * 2;
    q[j] = hval ? *(const u32x4*)(qp + off) : u32x4{0u, 0u, 0u, 0u};
  }
  // Blocks e .. e + 63, one a lane: place and scales.  Those that are done or whose pages
  // are not there have no bit in `left`.
  int at, e = first >> steps, sub = (first & ((1 << steps) - 1)) << 5;
  const int e1 = (end + (1 << steps) - 1) >> steps, cut = B - (((e1 << steps) - end) << 5);  // rows of the last block
  float ksc = 1.f, vsc = 1.f;
  uint64_t left = 0;
  auto look = [&]() {
    const int i = e + lane;
    at = i >= e1 ? -1 : (list ? list[i] : block_at(a, slot, g, i));
    if constexpr (KIND != kRowsBf16) {
      ksc = a.ks[max(at, 0)];
      vsc = a.vs[max(at, 0)];
    }
    left = __builtin_amdgcn_ballot_w64(at >= 0);
  };
  // to the next 32 rows; false: there are none
  auto next = [&]() {
    if (left && sub + 32 < (e + __builtin_ctzll(left) == e1 - 1 ? cut : B)) {
      sub += 32;
      return true;
    }
    sub = 0;
    left &= left - 1;
    while (!left && (e += 64) < e1) {
      look();
      settle(at);
      settle(ksc);
      settle(vsc);
    }
    return left != 0;
  };
  auto load_k = [&](const unsigned char* kp, u32x4 (&k0)[NK], u32x4 (&k1)[NK]) {
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      k0[j] = load_as<NT, u32x4>(kp + 64 * j);
      k1[j] = load_as<NT, u32x4>(kp + 16 * (D * E) + 64 * j);
    }
  };
  const int koff = l16 * (D * E) + 16 * lg, voff = 4 * lg * (D * E) + l16 * (VE * E);
  // the first of the 32 rows that are next, and a scale of theirs
  auto row = [&]() {
    return ((size_t)(uint32_t)__builtin_amdgcn_readlane(at, __builtin_ctzll(left)) << a.block_shift) + sub;
  };
  auto of = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), __builtin_ctzll(left))); };
  bool more = false;
  if (first < end) {
    look();
    more = left & 1;  // (the first block: from its row `sub` on)
    if (!more) {
      sub = 0;
      more = left != 0;
      if (!more) more = next();
    }
  }
  auto load_v = [&](size_t r, VRaw (&v)[8]) {
    const unsigned char* vp = a.cv + r * (D * E) + voff;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load_as<NT, VRaw>(vp + ((i < 4 ? 0 : 16) + (i & 3)) * (D * E));
  };
  u32x4 k0[NK], k1[NK];
  VRaw v[8];
  size_t r = 0;
  float xk = 1.f, xv = 1.f;
  if (more) {
    r = row();
    load_k(a.ck + r * (D * E) + koff, k0, k1);
    if (AHEAD) load_v(r, v);
    xk = of(ksc);
    xv = of(vsc);
  }
#pragma unroll
  for (int j = 0; j < D / 32; ++j) settle(q[j]);
  settle(ksc);
  settle(vsc);
  while (more) {
    // values of these rows, then keys of the next: the second product waits for the values
    // only
    if (!AHEAD) load_v(r, v);
    VRaw nv[8];
    const float xs = a.scale2 * xk, xlo = a.scale2_lo * xk, vs = xv;
    u32x4 n0[NK], n1[NK];
    more = next();
    if (more) {
      r = row();
      load_k(a.ck + r * (D * E) + koff, n0, n1);
      if (AHEAD) load_v(r, nv);
      xk = of(ksc);
      xv = of(vsc);
    }
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      if constexpr (KIND == kRowsBf16) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k0[j]), __builtin_bit_cast(bf16x8, q[j]), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k1[j]), __builtin_bit_cast(bf16x8, q[j]), s1, 0, 0, 0);
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 qq = __builtin_bit_cast(bf16x8, q[2 * j + u]);
          const u32x2 a0 = bf16x4<KIND>(k0[j][2 * u]), a1 = bf16x4<KIND>(k0[j][2 * u + 1]);
          const u32x2 b0 = bf16x4<KIND>(k1[j][2 * u]), b1 = bf16x4<KIND>(k1[j][2 * u + 1]);
          s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{a0[0], a0[1], a1[0], a1[1]}), qq, s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{b0[0], b0[1], b1[0], b1[1]}), qq, s1, 0, 0, 0);
        }
      }
    }
    const float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
    float pe[8];
    o.template softmax<KIND != kRowsBf16>(x, xs, xlo, vs, pe);
    if constexpr (KIND == kRowsInt8) {
      o.values8(pe, v);
    } else {
      uint32_t vw[8][VE / 2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (KIND == kRowsBf16) {
#pragma unroll
          for (int u = 0; u < VE / 2; ++u) vw[i][u] = v[i][u];
        } else {
#pragma unroll
          for (int u = 0; u < VE / 4; ++u) {
            const u32x2 w = bf16x4<KIND>(v[i][u]);
            vw[i][2 * u] = w[0];
            vw[i][2 * u + 1] = w[1];
          }
        }
      }
      o.template values<KIND == kRowsBf16>(pe, vw);
    }
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      k0[j] = n0[j];
      k1[j] = n1[j];
    }
    if (AHEAD)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = nv[i];
  }
}

// The first workgroups take a work item each, B / 32 a unit attend 32 rows each of the
// newest token's block, the last two a unit store a step's token: the longest first, so
// that the short ones fill the gaps.
template <int D, int KIND, bool NT>
__global__ __launch_bounds__(64) void block_attn(BlockArgs a) {
  constexpr int VE = D / 16;
  const int lane = tid() & 63, l16 = lane & 15, lg = lane >> 4, units = a.n * a.Hkv;
  const int parts = 1 << (a.block_shift - 5), item = bid_x(), w = item - a.max_items;
  if (w >= parts * units) {
    const int i = w - parts * units;
    put_token<D, KIND>(a, i >> 1, !(i & 1));
    return;
  }
  Soft<D> o;
  o.init();
  if (w >= 0) {
    const int unit = w / parts, r0 = w % parts * 32, b = unit / a.Hkv, g = unit % a.Hkv;
    const BlockSeq s = block_seq(a, b);
    const int at = s.tail && r0 <= (s.row & ((1 << a.block_shift) - 1)) ? uniform(block_at(a, s.slot, g, s.row >> a.block_shift)) : -1;
    if (at >= 0) attend_newest<D, KIND>(a, s, b, g, at, r0, o);
  } else {
    BlockCut c;
    if (!block_cut(a, item, true, c)) return;
    const int local = item - c.item0, g = local / c.items, chunk = local % c.items;
    const int nb = a.list ? a.list_ld : c.blocks;
    const int e0 = (int)((int64_t)chunk * nb / c.items), e1 = (int)((int64_t)(chunk + 1) * nb / c.items);
    attend_blocks<D, KIND, NT, false>(a, c.b, g, c.slot, a.list ? a.list + (size_t)(c.b * a.Hkv + g) * a.list_ld : nullptr,
                               e0 << (a.block_shift - 5), e1 << (a.block_shift - 5), o);
  }
  const float L = o.total();
  o.template by<KIND != kRowsBf16>(L > 0.f ? 1.f / L : 0.f);
  if (l16 >= a.G) return;
  const size_t pi = (size_t)(w < 0 ? parts * units + item : w) * a.G + l16;  // the units' parts of the newest block, then the items
  if (lg == 0) a.ml[pi] = make_float2(o.m, L);
  float* dst = a.part + pi * D + 4 * lg * VE;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int c = 0; c < VE; c += 4)
      *(f32x4*)(dst + e * VE + c) = f32x4{o.acc[c][e], o.acc[c + 1][e], o.acc[c + 2][e], o.acc[c + 3][e]};
}

// The same for short calls in one launch: a workgroup takes a whole unit, each wave a share
// of its 32-row steps, and joins them in LDS.
constexpr int kUnitWaves = 8;
template <int D, int KIND>
__global__ __launch_bounds__(64 * kUnitWaves) void block_attn_unit(BlockArgs a) {
  extern __shared__ __align__(16) float joins[];  // [kUnitWaves / 2][G][D]
  constexpr int VE = D / 16, W = kUnitWaves;
  __shared__ float2 mls[W][16];
  const int lane = tid() & 63, w = uniform(tid() >> 6), l16 = lane & 15, lg = lane >> 4, unit = bid_x();
  const int b = unit / a.Hkv, g = unit % a.Hkv, steps = a.block_shift - 5;
  const BlockSeq s = block_seq(a, b);
  if (s.slot < 0 || s.slot >= a.n_slots) {  // no rows: zeros
    if (w == 0 && l16 < a.G)
      for (int i = lg; i < D; i += 4) {
        const size_t oi = ((size_t)b * a.Hq + g * a.G + l16) * D + i;
        if (a.out_bf16) ((uint16_t*)a.out)[oi] = 0;
        else ((float*)a.out)[oi] = 0.f;
      }
    return;
  }
  const bool hval = l16 < a.G;
  const int nb = a.list ? a.list_ld : s.blocks, codes = nb << steps;
  const int at = s.tail ? uniform(block_at(a, s.slot, g, s.row >> a.block_shift)) : -1;
  const int total = codes + (at < 0 ? 0 : ((s.row & ((1 << a.block_shift) - 1)) >> 5) + 1);
  const int s0 = w * total / W, s1 = (w + 1) * total / W;
  Soft<D> o;
  o.init();
  if (s0 < codes)
    attend_blocks<D, KIND, false, true>(a, b, g, s.slot, a.list ? a.list + (size_t)unit * a.list_ld : nullptr, s0, min(s1, codes), o);
  if (KIND != kRowsBf16 && s0 < codes && codes < s1) o.by_total();
  for (int i = max(s0, codes); i < s1; ++i) attend_newest<D, KIND>(a, s, b, g, at, (i - codes) * 32, o);
  const float mine = o.total();
  if (lg == 0) mls[w][l16] = make_float2(o.m, mine);
  __syncthreads();
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) M = fmaxf(M, mls[i][l16].x);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float2 v = mls[i][l16];
    if (v.x != -INFINITY) L = fmaf(fast_exp2(v.x - M), v.y, L);
  }
  o.template by<KIND != kRowsBf16>(o.m == -INFINITY ? 0.f : fast_exp2(o.m - M) * (L > 0.f ? 1.f / L : 0.f));
  // the upper half of the waves hand theirs to the lower, until one has the sum
#pragma unroll
  for (int half = W / 2; half >= 1; half /= 2) {
    float* to = joins + ((w & (half - 1)) * a.G + l16) * D + 4 * lg * VE;
    if (w >= half && w < 2 * half && hval)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VE; c += 4)
          *(f32x4*)(to + e * VE + c) = f32x4{o.acc[c][e], o.acc[c + 1][e], o.acc[c + 2][e], o.acc[c + 3][e]};
    __syncthreads();
    if (w < half && hval)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VE; c += 4) {
          const f32x4 v = *(const f32x4*)(to + e * VE + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) o.acc[c + i][e] += v[i];
        }
    __syncthreads();
  }
  if (w == 0 && hval) {
    const size_t oi = ((size_t)b * a.Hq + g * a.G + l16) * D + 4 * lg * VE;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < VE; c += 4) {
        const f32x4 v = f32x4{o.acc[c][e], o.acc[c + 1][e], o.acc[c + 2][e], o.acc[c + 3][e]};
        if (a.out_bf16)
          *(u32x2*)((uint16_t*)a.out + oi + e * VE + c) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else
          *(f32x4*)((float*)a.out + oi + e * VE + c) = v;
      }
  }
  // (no wave reads the newest row but from the input, nor the block it may complete)
  if (a.k_new && (w == W - 1 || w == W - 2)) put_token<D, KIND>(a, unit, w == W - 1);
}

// ---------------------------------------------------------------- join
// A workgroup for each (sequence, query head): thread t takes dims 4 (t % DG) .. + 3 of
// items t / DG, t / DG + CL, ..., after the parts of the newest token's block.
constexpr int kJoinThreads = 256;
template <int D>
__global__ __launch_bounds__(kJoinThreads) void block_join(BlockArgs a) {
  constexpr int DG = D / 4, CL = kJoinThreads / DG, kHeld = 4;
  __shared__ f32x4 sacc[kJoinThreads];
  const int bh = bid_x(), b = bh / a.Hq, qh = bh % a.Hq, g = qh / a.G, h = qh % a.G, unit = b * a.Hkv + g;
  const int t = tid(), lane = t & 63, dg = t % DG, cl = t / DG;
  BlockCut c;
  if (!block_cut(a, b, false, c)) return;
  const int parts = (1 << a.block_shift) >> 5, items = c.items + parts, first = parts * a.n * a.Hkv + c.item0 + g * c.items - parts;
  auto place = [&](int i) { return (size_t)(i < parts ? parts * unit + i : first + i) * a.G + h; };
  // the first partials of the thread are in flight with the references
  f32x4 held[kHeld];
  float2 mheld[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const size_t pi = place(min(cl + j * CL, items - 1));
    held[j] = *(const f32x4*)(a.part + pi * D + 4 * dg);
    mheld[j] = a.ml[pi];
  }
  float m = -INFINITY, l = 0.f;
  for (int i = lane; i < items; i += 64) {
    const float2 v = a.ml[place(i)];
    const float mn = fmaxf(m, v.x);
    if (mn != -INFINITY) l = l * fast_exp2(m - mn) + v.y * fast_exp2(v.x - mn);
    m = mn;
  }
  float M = m;
#pragma unroll
  for (int x = 32; x >= 1; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
  const float L = warp_sum(m == -INFINITY ? 0.f : l * fast_exp2(m - M));
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  // the items' means by their shares: finite where the mean of all is (an item without a row
  // holds zeros)
  const float each = L > 0.f ? 1.f / L : 0.f;
  auto add = [&](f32x4 v, float2 i) { o += v * (i.x == -INFINITY ? 0.f : fast_exp2(i.x - M) * i.y * each); };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (cl + j * CL < items) add(held[j], mheld[j]);
#pragma unroll 4
  for (int i = cl + kHeld * CL; i < items; i += CL) {
    const size_t pi = place(i);
    add(*(const f32x4*)(a.part + pi * D + 4 * dg), a.ml[pi]);
  }
  sacc[t] = o;
  __syncthreads();
  if (cl) return;
#pragma unroll
  for (int i = 1; i < CL; ++i) o += sacc[dg + DG * i];
  const size_t oi = (size_t)bh * D + 4 * dg;
  if (a.out_bf16)
    *(u32x2*)((uint16_t*)a.out + oi) = u32x2{f32_to_bf16_bits(o[0]) | (f32_to_bf16_bits(o[1]) << 16),
                                             f32_to_bf16_bits(o[2]) | (f32_to_bf16_bits(o[3]) << 16)};
  else
    *(f32x4*)((float*)a.out + oi) = o;
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }
int kind_of(int kv_dtype) { return kv_dtype == SNAP_BF16 ? kRowsBf16 : (kv_dtype == SNAP_INT8 ? kRowsInt8 : kRowsFp8); }

BlockArgs block_args(const snap_params& p, const snap_block_cache& c, const int32_t* rows, int n, const int32_t* slot_ids,
                     const void* k_new, const void* v_new) {
  BlockArgs a = {};
  a.ck = (unsigned char*)c.k;
  a.cv = (unsigned char*)c.v;
  a.ks = c.k_scale;
  a.vs = c.v_scale;
  a.kt = (unsigned char*)c.k_tail;
  a.vt = (unsigned char*)c.v_tail;
  a.bound = (int8_t*)c.bound;
  a.bscale = c.bound_scale;
  a.rows = rows;
  a.slot_ids = slot_ids;
  a.table = c.page_table;
  a.k_new = k_new;
  a.v_new = v_new;
  a.n = n;
  a.Hq = p.n_q_heads;
  a.Hkv = p.n_kv_heads;
  a.G = p.n_q_heads / p.n_kv_heads;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = log2_of(c.page_size);
  a.block_shift = log2_of(c.block);
  a.max_pages = c.max_pages;
  return a;
}

}  // namespace

SNAP_DEBUG_READER(debug_flags_blocks)

// ---------------------------------------------------------------- host side
int block_chosen(const snap_params& p, int block) {
  return (p.sink + block - 1) / block + (p.recent - 1 + block - 1) / block + (p.topk + block - 1) / block;
}

// Work items that the card holds at once, by the registers of a wave (two a SIMD).
constexpr int kResident = 2048;
BlockGeometry block_geometry(const snap_params& p, int n, int max_rows, int block, bool select) {
  BlockGeometry g{};
  const int units = (n > 0 ? n : 1) * p.n_kv_heads, G = p.n_q_heads / p.n_kv_heads;
  g.blocks = max_rows / block;
  g.chosen = block_chosen(p, block);
  const int most = g.blocks < 1 ? 1 : g.blocks;
  g.list_ld = g.chosen < most ? (g.chosen < 1 ? 1 : g.chosen) : most;
  (PagedCut&)g = paged_cut(units, kResident, (int64_t)units * most);
  size_t items = (size_t)units * (block / 32) + g.max_items;
  if (select) {  // the same items for every unit
    // Of 128-wide rows, which keep more bytes in flight a wave, half the card's waves are
    // enough, with half the partials to join.  All / half of them, 8 KV heads, us a call:
    // 128 int8 16 x 4096 rows 55.9/54.2, 8 x 4096 36.9/35.2, 4 x 30000 66.0/62.8, 32 x 4096
    // 78.0/78.9, bf16 16 x 4096 65.2/63.1, E4M3 16 x 2000 40.6/39.8; 64 E4M3 64 x 7500
    // 122/149.
    int each = (p.d_qk == 128 ? kResident / 2 : kResident) / units;
    each = each < 1 ? 1 : (each > g.list_ld ? g.list_ld : each);
    g.max_items = units * each;
    // (a bound that does not fall as sequences or rows grow, and serves calls without)
    const int64_t bound = units > kResident ? units : kResident;
    items += (size_t)((int64_t)units * most < bound ? (int64_t)units * most : bound);
  }
  size_t off = 0;
  g.off_part = off;
  off = align256(off + items * G * p.d_v * sizeof(float));
  g.off_ml = off;
  off = align256(off + items * G * sizeof(float2));
  g.off_list = off;
  if (select) off = align256(off + (size_t)units * g.list_ld * sizeof(int32_t));
  g.off_keys = off;
  if (select) off = align256(off + (size_t)units * most * sizeof(uint32_t));
  g.bytes = off;
  return g;
}

// Whether a unit's blocks are scored by a launch of their own, kBatch of them a workgroup,
// or by the one workgroup that chooses among them.  That one takes in 30 to 50 bytes a
// nanosecond; the launch costs 3 to 5 us.  Whole calls, 8 KV heads, one launch / two, us:
//   bounds a unit           128 KB      256 KB      512 KB      1 MB
//   d 128     1 sequence   19.1/20.6   22.0/21.6   26.9/22.4   36.5/24.3
//             4            21.8/23.8   24.7/24.8   31.6/26.6   43.7/32.4
//             8            24.8/27.0   28.2/28.7   34.4/33.0   46.7/44.3
//            12            27.5/30.0   30.9/33.6   37.6/39.4   50.9/52.9
//            16            30.2/33.1   33.9/37.1   42.0/49.1   58.4/61.4
//            32            46.0/49.9   50.5/61.6   64.8/73.2   97.3/99.7
//   d 64      1            19.1/21.4   22.8/22.2   30.2/23.7
//             4            21.3/23.9   25.6/25.6   36.1/28.0
//             8            23.5/26.0   29.1/28.1   38.5/33.1
//            12            26.0/28.3   30.8/32.5   41.1/38.7
//            16            26.8/29.9   32.6/34.4   43.3/42.9
//            32            34.0/37.6   41.8/45.4   62.0/59.1
// (Where the rule takes one, 64-wide rows are 1 to 6% faster by two at 512 KB from 12
// sequences on, and 3% at 256 KB of one or eight.)
// (Past 8192 blocks the one that scores would not have its keys in LDS.)
static bool scored_apart(const snap_params& p, int units, int blocks) {
  return units <= 64 ? (size_t)blocks * 2 * p.d_qk >= (size_t)512 << 10 : blocks > 4096;
}

// Whether a workgroup of eight waves takes a whole unit, so that one launch does: with
// few units while a wave has two steps of 32 rows (64-wide) or one, with 128 while it has
// four, with enough units to fill the card while it has eight, or 16 of 128 bytes a row
// (then nothing is written for the join).  Measured, one launch / two, 32 query heads on 8,
// us of a replayed call:
//   rows                250         500        1000        2000        3900
//   128 int8   1 x   8.8/10.1  10.4/10.1  14.1/10.2  20.5/10.6   33.2/11.9
//             16     9.0/11.5  11.5/12.6  15.9/16.4  22.4/21.5   36.1/30.2
//             32    10.5/13.2  13.6/16.7  18.3/22.2  28.5/32.5   54.1/53.1
//             64    19.0/19.0  24.6/24.6  34.4/35.0  60.4/58.2    104/94.4
//   128 bf16   1     8.7/9.6   11.0/9.6   16.9/9.7   24.6/10.3   41.4/12.3
//             16     9.5/11.6  12.8/14.4  19.1/19.7  28.3/30.8   59.3/49.1
//             32    11.8/14.4  16.4/20.0  25.7/32.5  51.6/51.1   94.4/91.1
//             64    21.3/21.7  30.4/34.6  57.9/54.8   100/94.7    182/168
//   64 int8    1     6.5/8.5    8.1/8.6   10.2/8.6   14.8/9.0    23.5/11.1
//             16     6.6/9.7    8.3/11.0  11.2/12.7  16.5/15.5   25.3/20.3
//             32     6.8/11.5   9.2/13.5  12.8/16.0  17.6/20.6   26.9/29.7
//             64     9.5/15.4  13.7/18.1  18.9/22.6  28.5/32.2   54.0/53.2
//   64 bf16    1     6.7/8.4    8.2/8.5   11.1/8.6   16.1/8.9    26.2/11.2
//             16     6.9/9.8    8.7/11.3  12.7/14.8  17.9/19.4   28.7/28.0
//             32     7.7/11.8  11.5/15.7  16.3/19.9  24.9/29.1   49.2/49.1
//             64    11.4/17.7  16.6/22.7  25.3/31.8  50.3/55.0   91.4/95.1
// Against the rule, by 4 to 9%: 1000 (bf16) and 2000 128-wide rows of 64 sequences, which
// two launches take faster; 2000 bf16 rows of 16 sequences and 3900 64-wide ones of 64,
// which one does.
// The rule goes by the bound of the rows, not by the rows that are there: a far one takes
// two launches.
// (calls that are not replayed cost the host 9 us with one launch, 11 with two)
static bool whole_units(const snap_params& p, int units, int blocks, int block) {
  const int row_bytes = 2 * p.d_qk * (p.kv_dtype == SNAP_BF16 ? 2 : 1);
  const int share = units >= 256 ? (row_bytes > 128 ? 8 : 16) : (units >= 128 ? 4 : (p.d_qk == 64 ? 2 : 1));
  return (int64_t)blocks * (block / 32) <= share * kUnitWaves;
}

snap_status launch_block_append(const snap_params& p, const snap_block_cache& c, const int32_t* rows, int n,
                                const int32_t* slot_ids, const int32_t* lengths, const int32_t* starts, int tokens,
                                int max_len, const void* k_new, const int64_t* k_stride, const void* v_new,
                                const int64_t* v_stride, hipStream_t stream) {
  BlockAppend a = {};
  a.c = block_args(p, c, rows, n, slot_ids, k_new, v_new);
  a.lengths = lengths;
  a.starts = starts;
  a.tokens = tokens;
  a.max_len = max_len;
  const int64_t d = p.d_qk, h = p.n_kv_heads;
  const int64_t kd[3] = {h * max_len * d, starts ? d : max_len * d, starts ? h * d : d};
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = 2 * (k_stride ? k_stride[i] : kd[i]);
    a.vs[i] = 2 * (v_stride ? v_stride[i] : kd[i]);
  }
  const int blocks = (int)(((int64_t)max_len + 2 * c.block - 2) / c.block);
#define SNAP_BLOCK_APPEND(D, KIND) {block_append<D, KIND, 32>, block_append<D, KIND, 64>, block_append<D, KIND, 128>}
  static constexpr void (*kernels[2][3][3])(BlockAppend) = {  // [width][rows][block]
      {SNAP_BLOCK_APPEND(64, kRowsBf16), SNAP_BLOCK_APPEND(64, kRowsFp8), SNAP_BLOCK_APPEND(64, kRowsInt8)},
      {SNAP_BLOCK_APPEND(128, kRowsBf16), SNAP_BLOCK_APPEND(128, kRowsFp8), SNAP_BLOCK_APPEND(128, kRowsInt8)}};
#undef SNAP_BLOCK_APPEND
  hipLaunchKernelGGL(kernels[p.d_qk == 128][kind_of(p.kv_dtype)][a.c.block_shift - 5], dim3(1 + blocks / 2, p.n_kv_heads, n),
                     dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

snap_status launch_block_decode(const snap_params& p, const snap_block_cache& c, const int32_t* rows, int n,
                                const int32_t* slot_ids, int max_rows, const void* q, const void* k_new, const void* v_new,
                                void* out, int out_dtype, bool select, int32_t* sel_out, void* ws, hipStream_t stream) {
  const BlockGeometry geo = block_geometry(p, n, max_rows, c.block, select);
  BlockArgs a = block_args(p, c, rows, n, slot_ids, k_new, v_new);
  a.q = q;
  a.part = (float*)((unsigned char*)ws + geo.off_part);
  a.ml = (float2*)((unsigned char*)ws + geo.off_ml);
  a.out = out;
  a.max_rows = max_rows;
  a.waves = geo.waves;
  a.target = geo.target;
  a.max_items = geo.max_items;
  a.chosen = geo.chosen;
  a.list_ld = geo.list_ld;
  a.out_bf16 = out_dtype == SNAP_BF16;
  split_scale2(p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_qk), a.scale2, a.scale2_lo);
  const int units = n * p.n_kv_heads;
  if (select) {
    a.list = (int32_t*)((unsigned char*)ws + geo.off_list);
    a.sel_out = sel_out;
    a.sink = p.sink;
    a.recent = p.recent;
    a.best = (p.topk + c.block - 1) / c.block;
    const bool apart = scored_apart(p, units, geo.blocks);
    if (apart) {
      a.keys = (uint32_t*)((unsigned char*)ws + geo.off_keys);
      a.key_ld = geo.blocks;
      const int chunk = p.d_qk == 128 ? BlockScores<128, kScoreThreads / 64>::kBatch : BlockScores<64, kScoreThreads / 64>::kBatch;
      hipLaunchKernelGGL((p.d_qk == 128 ? block_score<128> : block_score<64>), dim3((geo.blocks + chunk - 1) / chunk, units),
                         dim3(kScoreThreads), 0, stream, a);
      if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
    }
    const size_t lds = (size_t)(geo.blocks < 1 ? 1 : geo.blocks) * sizeof(uint32_t);
    static constexpr void (*choose[2][2])(BlockArgs) = {{block_select<64, false>, block_select<64, true>},
                                                        {block_select<128, false>, block_select<128, true>}};
    hipLaunchKernelGGL(choose[p.d_qk == 128][apart], dim3(units), dim3(kSelThreadsB), lds, stream, a);
    if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  }
  if (whole_units(p, units, select ? geo.list_ld : geo.blocks, c.block)) {
    static constexpr void (*kernels[2][3])(BlockArgs) = {
        {block_attn_unit<64, kRowsBf16>, block_attn_unit<64, kRowsFp8>, block_attn_unit<64, kRowsInt8>},
        {block_attn_unit<128, kRowsBf16>, block_attn_unit<128, kRowsFp8>, block_attn_unit<128, kRowsInt8>}};
    hipLaunchKernelGGL(kernels[p.d_qk == 128][kind_of(p.kv_dtype)], dim3(units), dim3(64 * kUnitWaves),
                       (size_t)(kUnitWaves / 2) * a.G * p.d_v * sizeof(float), stream, a);
    return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
  }
  // streaming loads where the blocks read are more than half the last-level cache
  const size_t row_bytes = (size_t)2 * p.d_qk * (p.kv_dtype == SNAP_BF16 ? 2 : 1);
  const size_t call_bytes = (size_t)units * (select ? geo.list_ld : geo.blocks) * c.block * row_bytes;
  const bool nt = p.kv_reuse == SNAP_KV_STREAM || (p.kv_reuse == SNAP_KV_AUTO && call_bytes >= (size_t)128 << 20);
#define SNAP_BLOCK_ATTN(D) \
  {{block_attn<D, kRowsBf16, false>, block_attn<D, kRowsFp8, false>, block_attn<D, kRowsInt8, false>}, \
   {block_attn<D, kRowsBf16, true>, block_attn<D, kRowsFp8, true>, block_attn<D, kRowsInt8, true>}}
  static constexpr void (*kernels[2][2][3])(BlockArgs) = {SNAP_BLOCK_ATTN(64), SNAP_BLOCK_ATTN(128)};  // [width][NT][rows]
#undef SNAP_BLOCK_ATTN
  hipLaunchKernelGGL(kernels[p.d_qk == 128][nt][kind_of(p.kv_dtype)], dim3(units * ((k_new ? 2 : 0) + c.block / 32) + geo.max_items),
                     dim3(64), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  hipLaunchKernelGGL((p.d_qk == 128 ? block_join<128> : block_join<64>), dim3(n * p.n_q_heads), dim3(kJoinThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

}  // namespace snap
