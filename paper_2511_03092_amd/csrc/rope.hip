// rope.hip -- rotary positions (Sec. III-B: keys are cached after positional
// encoding and never re-encoded): q and k heads turned pair by pair, from the
// layout a projection leaves them in to the one the attention calls take.
//
// Angles.  position * f is up to 2^31 radians and only its fraction of a turn
// matters, so the product, its rounding to a quarter turn and the remainder are
// formed in 64 bits, with what the product's rounding loses and the low part of f
// added to the remainder: together off by under 2^-29 turns at the farthest position
// (f's own 2^-58), where 64 bits alone are off by 2^-24.3.  Sine and cosine of the
// remainder, at most an eighth of a turn, are then Taylor sums in 32 bits: the terms
// left out are under 2^-29 (x^11 / 11! and x^12 / 12! at pi/4).
#include <math.h>

#include "snap_internal.h"

namespace snap {

struct RopeArgs {
  const void* x[2];
  void* y[2];
  int64_t xs[2][3], ys[2][3];  // sequence, head, token strides (elements)
  int heads[2];
  int n, max_len, d, rot_start, rot, pairs, n_slots, in_place, slices;
  const int32_t* pos;
  const int32_t* slot_ids;
  const int32_t* lengths;
  float amp;
  // turns a position of each pair, in two terms (the second in 32 bits: with 16 bytes a
  // pair a prompt of 4000 tokens takes 17.0 us instead of 15.4)
  double turns[kRopeMaxPairs];
  float turns_lo[kRopeMaxPairs];
};

// amp * (cos, sin) of the position's turns
__device__ __forceinline__ void turn_of(double position, double per, float per_lo, float amp, float& c, float& s) {
  const double turns = position * per, rest = __builtin_fma(position, (double)per_lo, __builtin_fma(position, per, -turns));
  // |turns| * 4 < 2^34, so added to 1.5 * 2^52 it is rounded to a whole number of
  // quarters, whose last two bits are the sum's
  const double sum = __builtin_fma(turns, 4.0, 0x1.8p52), quarter = sum - 0x1.8p52;
  const int q = (int)(__builtin_bit_cast(uint64_t, sum) & 3u);
  const float x = (float)((__builtin_fma(-0.25, quarter, turns) + rest) * 6.283185307179586476925);
  const float x2 = x * x;
  float sn = fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);  // 1/9!, -1/7!
  sn = fmaf(x2, sn, 8.3333333e-3f);
  sn = fmaf(x2, sn, -1.6666667e-1f);
  sn = fmaf(x * x2, sn, x);
  float cs = fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);  // -1/10!, 1/8!
  cs = fmaf(x2, cs, -1.3888889e-3f);
  cs = fmaf(x2, cs, 4.1666667e-2f);
  cs = fmaf(x2, cs, -0.5f);
  cs = fmaf(x2, cs, 1.f);
  const float a = (q & 1) ? sn : cs, b = (q & 1) ? cs : sn;
  c = amp * ((q == 1 || q == 2) ? -a : a);
  s = amp * (q >= 2 ? -b : b);
}

// The token of flat index i: its sequence, whether it is there, its position.
struct RopeToken {
  int b, t;
  bool live;
  double position;
};
__device__ __forceinline__ RopeToken rope_token(const RopeArgs& a, unsigned i) {
  RopeToken k;
  k.b = (int)(i / (unsigned)a.max_len);
  k.t = (int)(i - (unsigned)k.b * (unsigned)a.max_len);
  k.live = !a.lengths || k.t < a.lengths[k.b];
  int start = 0;
  if (a.pos) {
    const int slot = a.slot_ids[k.b];
    if (slot < 0 || slot >= a.n_slots)
      k.live = false;
    else
      start = a.pos[slot];
  }
  k.position = (double)start + (double)k.t;
  return k;
}

template <typename T>
__device__ __forceinline__ float rope_get(const T* p) {
  if constexpr (sizeof(T) == 2)
    return bf16_bits_to_f32(*p);
  else
    return *p;
}
template <typename T>
__device__ __forceinline__ void rope_set(T* p, float v) {
  if constexpr (sizeof(T) == 2)
    *p = (uint16_t)f32_to_bf16_bits(v);
  else
    *p = v;
}

// One 16-byte piece (halves: a piece of the first half and its partner of the
// second) of a token per thread, over the heads of a slice: the angles are formed
// once and turn every head.  Copied dims take threads of their own.  HBM bound: four
// heads' pieces are loaded before the first is turned, and the token's share of
// every head is read by the same threads, so that both a token-by-token input and a
// head-by-head output move in whole 128-byte lines.
constexpr int kRopeHeads = 4;

template <typename T>
struct RopePiece {
  static constexpr int E = 16 / sizeof(T);
  float v[E];
  __device__ __forceinline__ void unpack(u32x4 raw) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        v[2 * i] = __uint_as_float(raw[i] << 16);
        v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
      } else {
        v[i] = __uint_as_float(raw[i]);
      }
    }
  }
  __device__ __forceinline__ u32x4 pack() const {
    u32x4 raw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2)
        raw[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
      else
        raw[i] = __float_as_uint(v[i]);
    }
    return raw;
  }
};

template <typename T, bool PAIRS>
__global__ __launch_bounds__(256) void rope_pieces(RopeArgs a) {
  constexpr int E = RopePiece<T>::E, NA = PAIRS ? E / 2 : E;  // angles of a thread
  const unsigned nc = a.rot / (PAIRS ? E : 2 * E), cols = nc + (a.in_place ? 0 : (a.d - a.rot) / E);
  const unsigned i = (unsigned)bid_x() * 256u + (unsigned)tid();
  const unsigned tok = i / cols, col = i % cols;
  if (tok >= (unsigned)a.n * (unsigned)a.max_len) return;
  const RopeToken k = rope_token(a, tok);
  if (!k.live) return;
  const bool turn = col < nc;
  float c[NA], s[NA];
  int d1, d2 = 0;
  if (turn) {
#pragma unroll
    for (int e = 0; e < NA; ++e) turn_of(k.position, a.turns[col * NA + e], a.turns_lo[col * NA + e], a.amp, c[e], s[e]);
    d1 = a.rot_start + col * E;
    d2 = d1 + a.rot / 2;
  } else {
    d1 = (col - nc) * E;
    if (d1 >= a.rot_start) d1 += a.rot;
  }
  const int total = a.heads[0] + a.heads[1];
  for (int h0 = bid_y(); h0 < total; h0 += kRopeHeads * a.slices) {
    u32x4 r1[kRopeHeads], r2[kRopeHeads];
#pragma unroll
    for (int u = 0; u < kRopeHeads; ++u) {
      const int h = h0 + u * a.slices;
      if (h >= total) break;
      const int o = h < a.heads[0] ? 0 : 1, hh = o ? h - a.heads[0] : h;
      const T* x = (const T*)a.x[o] + k.b * a.xs[o][0] + hh * a.xs[o][1] + k.t * a.xs[o][2];
      r1[u] = *(const u32x4*)(x + d1);
      if (!PAIRS && turn) r2[u] = *(const u32x4*)(x + d2);
    }
#pragma unroll
    for (int u = 0; u < kRopeHeads; ++u) {
      const int h = h0 + u * a.slices;
      if (h >= total) break;
      const int o = h < a.heads[0] ? 0 : 1, hh = o ? h - a.heads[0] : h;
      T* y = (T*)a.y[o] + k.b * a.ys[o][0] + hh * a.ys[o][1] + k.t * a.ys[o][2];
      if (!turn) {
        *(u32x4*)(y + d1) = r1[u];
        continue;
      }
      RopePiece<T> p, q;
      p.unpack(r1[u]);
      if constexpr (PAIRS) {
#pragma unroll
        for (int e = 0; e < NA; ++e) {
          const float x1 = p.v[2 * e], x2 = p.v[2 * e + 1];
          p.v[2 * e] = fmaf(x1, c[e], -(x2 * s[e]));
          p.v[2 * e + 1] = fmaf(x2, c[e], x1 * s[e]);
        }
      } else {
        q.unpack(r2[u]);
#pragma unroll
        for (int e = 0; e < NA; ++e) {
          const float x1 = p.v[e], x2 = q.v[e];
          p.v[e] = fmaf(x1, c[e], -(x2 * s[e]));
          q.v[e] = fmaf(x2, c[e], x1 * s[e]);
        }
        *(u32x4*)(y + d2) = q.pack();
      }
      *(u32x4*)(y + d1) = p.pack();
    }
  }
}

// The same for pieces that are not whole: rotated dims, widths, strides or
// addresses that 16 bytes do not divide.  One pair or copied dim per thread, so bound by
// the number of accesses: the 32k prompt with 24 of its 128 dims rotated takes 475 us
// (whole pieces, all 128: 142).
template <typename T>
__global__ __launch_bounds__(256) void rope_any(RopeArgs a) {
  const unsigned np = a.rot / 2, cols = np + (a.in_place ? 0 : a.d - a.rot);
  const unsigned i = (unsigned)bid_x() * 256u + (unsigned)tid();
  const unsigned tok = i / cols, col = i % cols;
  if (tok >= (unsigned)a.n * (unsigned)a.max_len) return;
  const RopeToken k = rope_token(a, tok);
  if (!k.live) return;
  int d1, d2 = -1;
  float c = 1.f, s = 0.f;
  if (col < np) {
    d1 = a.rot_start + (a.pairs ? 2 * col : col);
    d2 = d1 + (a.pairs ? 1 : np);
    turn_of(k.position, a.turns[col], a.turns_lo[col], a.amp, c, s);
  } else {
    d1 = col - np;
    if (d1 >= a.rot_start) d1 += a.rot;
  }
  for (int h = bid_y(); h < a.heads[0] + a.heads[1]; h += a.slices) {
    const int o = h < a.heads[0] ? 0 : 1, hh = o ? h - a.heads[0] : h;
    const T* x = (const T*)a.x[o] + k.b * a.xs[o][0] + hh * a.xs[o][1] + k.t * a.xs[o][2];
    T* y = (T*)a.y[o] + k.b * a.ys[o][0] + hh * a.ys[o][1] + k.t * a.ys[o][2];
    if (d2 < 0) {
      y[d1] = x[d1];
    } else {
      const float x1 = rope_get(x + d1), x2 = rope_get(x + d2);
      rope_set(y + d1, fmaf(x1, c, -(x2 * s)));
      rope_set(y + d2, fmaf(x2, c, x1 * s));
    }
  }
}

// ---------------------------------------------------------------- host side
// Turns a position of every pair, by the rule (64 bits and more: far positions
// multiply them by up to 2^31).
static void rope_turns(const snap_rope_params& r, double* out, float* lo_out) {
  const int np = r.rot_dim / 2;
  const long double two_pi = 6.283185307179586476925286766559L;
  const long double step = powl((long double)r.base, -2.0L / r.rot_dim);
  double lo = 0, hi = 0;
  if (r.rule == SNAP_ROPE_BY_INDEX) {
    const double per = r.rot_dim / (2.0 * log((double)r.base)), circle = 6.283185307179586476925;
    lo = fmax(0.0, floor(per * log(r.orig_len / (circle * r.high_turns))));
    hi = fmin(r.rot_dim - 1.0, ceil(per * log(r.orig_len / (circle * r.low_turns))));
  }
  long double f = 1.0L;
  for (int i = 0; i < np; ++i, f *= step) {
    long double w = 1.0L;  // share of the unchanged frequency
    if (r.rule == SNAP_ROPE_DIVIDE) {
      w = 0.0L;
    } else if (r.rule == SNAP_ROPE_BY_TURNS) {
      w = (r.orig_len * f / two_pi - r.low_turns) / ((long double)r.high_turns - r.low_turns);
    } else if (r.rule == SNAP_ROPE_BY_INDEX) {
      w = 1.0L - (i - lo) / fmax(hi - lo, 0.001);
    }
    w = w < 0 ? 0 : (w > 1 ? 1 : w);
    const long double g = w == 1.0L ? f : w * f + (1.0L - w) * f / r.factor;
    out[i] = (double)(g / two_pi);
    lo_out[i] = (float)(g / two_pi - out[i]);
  }
}

snap_status launch_rope(const snap_rope_params& r, int dtype, int n_seq, int max_len, int d, const int32_t* pos,
                        int n_slots, const int32_t* slot_ids, const int32_t* lengths, const snap_rope_heads* q,
                        const snap_rope_heads* k, hipStream_t stream) {
  if (k && r.rot_dim < d && (q->x == q->y) != (k->x == k->y)) {
    // Of the operand in place only the rotated dims are touched: a launch each.  (Bounds
    // of the copied heads in the kernels took the 32k prompt from 142 to 157 us and more.)
    const snap_status st = launch_rope(r, dtype, n_seq, max_len, d, pos, n_slots, slot_ids, lengths, q, nullptr, stream);
    if (st != SNAP_OK) return st;
    return launch_rope(r, dtype, n_seq, max_len, d, pos, n_slots, slot_ids, lengths, k, nullptr, stream);
  }
  RopeArgs a = {};
  const snap_rope_heads* op[2] = {q, k};
  bool in_place = true;
  for (int o = 0; o < 2; ++o) {
    if (!op[o]) continue;
    a.x[o] = op[o]->x;
    a.y[o] = op[o]->y;
    a.heads[o] = op[o]->n_heads;
    const int size[3] = {n_seq, op[o]->n_heads, max_len};
    for (int i = 0; i < 3; ++i) {  // (a stride along a size of 1 says nothing)
      a.xs[o][i] = size[i] > 1 ? op[o]->x_stride[i] : 0;
      a.ys[o][i] = size[i] > 1 ? op[o]->y_stride[i] : 0;
    }
    in_place = in_place && op[o]->x == op[o]->y;
  }
  a.n = n_seq;
  a.max_len = max_len;
  a.d = d;
  a.rot_start = r.rot_start;
  a.rot = r.rot_dim;
  a.pairs = r.layout == SNAP_ROPE_PAIRS;
  a.n_slots = n_slots;
  a.in_place = in_place;
  a.pos = pos;
  a.slot_ids = slot_ids;
  a.lengths = lengths;
  a.amp = r.amplitude;
  rope_turns(r, a.turns, a.turns_lo);
  const int E = dtype == SNAP_F32 ? 4 : 8;
  bool whole = (d | r.rot_start | (a.pairs ? r.rot_dim : r.rot_dim / 2)) % E == 0;
  for (int o = 0; o < 2; ++o) {
    whole = whole && (((uintptr_t)a.x[o] | (uintptr_t)a.y[o]) & 15u) == 0;
    for (int i = 0; i < 3; ++i) whole = whole && (a.xs[o][i] | a.ys[o][i]) % E == 0;
  }
  const int turned = whole ? (a.pairs ? a.rot / E : a.rot / (2 * E)) : a.rot / 2;
  const int64_t threads = (int64_t)n_seq * max_len * (turned + (in_place ? 0 : (d - a.rot) / (whole ? E : 1)));
  // heads split over workgroups until 16 waves a CU have work
  const int heads = a.heads[0] + a.heads[1];
  const int64_t want = ((int64_t)4096 * 64 + threads - 1) / threads;
  a.slices = (int)(want > heads ? heads : want);
  if (a.slices > 65535) a.slices = 65535;
  const dim3 grid((unsigned)((threads + 255) / 256), (unsigned)a.slices);
  void (*f)(RopeArgs);
  if (!whole)
    f = dtype == SNAP_BF16 ? rope_any<uint16_t> : rope_any<float>;
  else if (a.pairs)
    f = dtype == SNAP_BF16 ? rope_pieces<uint16_t, true> : rope_pieces<float, true>;
  else
    f = dtype == SNAP_BF16 ? rope_pieces<uint16_t, false> : rope_pieces<float, false>;
  hipLaunchKernelGGL(f, grid, dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

}  // namespace snap
