// evict.hip -- eviction from the paged cache by accumulated attention weight.
//
//   evict_pick     one workgroup per (sequence, KV head): the weight of the last
//                  row kept (radix select over the weights' bits), then the rows
//                  to move and where to, in ascending order of both
//   evict_split_*  the same in two launches, for more rows
//   evict_move     copies those rows; sources lie from the budget on and
//                  destinations below it, so no row is both
#include "snap_internal.h"

namespace snap {

namespace {

struct EvictArgs {
  unsigned char* ck;
  unsigned char* cv;
  int32_t* token;
  float* weight;
  const int32_t* rows;
  const int32_t* pos;
  int32_t* rows_out;
  const int32_t* slot_ids;
  const int32_t* table;
  int32_t* kept_out;
  int32_t* count;  // [units] moves
  int32_t* src;    // [units][max_moves]
  int32_t* dst;
  int Hkv, n_slots, n_pages, page_shift, max_pages, max_rows, budget, sink, recent, max_moves, kbytes, vbytes;
};

__device__ __forceinline__ int64_t evict_row(const EvictArgs& a, int slot, int g, int r) {
  const int page = a.table[(size_t)slot * a.max_pages + (r >> a.page_shift)];
  if (page < 0 || page >= a.n_pages) return -1;
  return (((int64_t)page * a.Hkv + g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
}

// A row's rank among those that are not protected: one more than its weight's bits
// (weights are not negative, so their bits are in their order; NaN and negative: 0).
__device__ __forceinline__ uint32_t weight_key(uint32_t bits) { return bits > 0x7f800000u ? 1u : bits + 1u; }

// ---------------------------------------------------------------- selection
// A row that is to be kept whatever its weight: above every weight's bits.
constexpr uint32_t kProtected = 0xffffffffu;
// A row past those looked at or in a page that is not there: below every weight's, so
// that it is never counted to nor kept.  Where such a row lies below the budget there is
// one place less to keep rows in, and nothing moves into it.
constexpr uint32_t kAbsent = 0;
constexpr int kPickThreads = 1024;
constexpr int kPickWaves = kPickThreads / 64;
constexpr int kTileRows = 4 * kPickThreads;  // four neighbouring rows (of one page) a thread
constexpr int kPickRows = 2 * kTileRows;     // rows that one workgroup selects among
// The keys' 31 bits (but for kProtected) in three parts, the leading ones (exponent and
// three bits more) first.
constexpr int kParts = 3;
constexpr int kBins = 2048;
__device__ __forceinline__ constexpr int part_shift(int part) { return part == 0 ? 20 : (part == 1 ? 10 : 0); }
__device__ __forceinline__ constexpr int part_bins(int part) { return part == 0 ? 2048 : 1024; }

typedef int i32x4 __attribute__((ext_vector_type(4)));

// A unit's rows and counters: R rows that the call looks at, `left` the slot's counter
// after it (a counter below zero stays; rows past max_rows count).
struct EvictUnit {
  int unit, slot, g, R, left, late;
};
__device__ __forceinline__ bool evict_unit(const EvictArgs& a, int unit, EvictUnit& u) {
  const int b = unit / a.Hkv;
  u.unit = unit;
  u.g = unit % a.Hkv;
  u.slot = a.slot_ids[b];
  if (u.slot < 0 || u.slot >= a.n_slots) return false;
  const int held = a.rows[u.slot];
  u.R = held < 0 ? 0 : (held > a.max_rows ? a.max_rows : held);
  u.left = held < a.budget ? held : a.budget;
  u.late = a.pos[u.slot] - a.recent;
  return true;
}

// What kept_out says of row r of a unit that is left as it is.
__device__ __forceinline__ int kept_in_place(const EvictArgs& a, const EvictUnit& u, int r) {
  return r < u.left && r < a.max_pages << a.page_shift && evict_row(a, u.slot, u.g, r) >= 0 ? r : -1;
}

// The keys of this thread's four rows of N tiles from row r0 on.
// No load stands behind a branch: rows that are not there are read at row 0 of page
// 0, so that every page id, and then every row, is in flight at once.
template <int N>
__device__ __forceinline__ void load_keys(const EvictArgs& a, const EvictUnit& u, int r0, uint32_t (&key)[N][4]) {
  int page[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int r = min(r0 + j * kTileRows + 4 * tid(), u.R - 1);
    page[j] = a.table[(size_t)u.slot * a.max_pages + (r >> a.page_shift)];
  }
  i32x4 tok[N];
  u32x4 w[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int r = r0 + j * kTileRows + 4 * tid();
    if (page[j] >= a.n_pages || r >= u.R) page[j] = -1;
    const int64_t row = page[j] < 0 ? 0 : (((int64_t)page[j] * a.Hkv + u.g) << a.page_shift) + (r & ((1 << a.page_shift) - 1));
    tok[j] = *(const i32x4*)(a.token + row);
    w[j] = *(const u32x4*)(a.weight + row);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      key[j][e] = page[j] < 0 || r0 + j * kTileRows + 4 * tid() + e >= u.R ? kAbsent
                  : tok[j][e] < a.sink || tok[j][e] >= u.late             ? kProtected
                                                                          : weight_key(w[j][e]);
}

// Sums of N values over the workgroup (every thread calls; red: N ints a wave).
template <int N>
__device__ __forceinline__ void block_sums(int (&v)[N], int* red) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_total(v[i]);
  __syncthreads();
  if ((tid() & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[(tid() >> 6) * N + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) v[i] += red[w * N + i];
  }
}

// The bin of a part's histogram that holds the rem-th largest, and how many are in
// the bins above it; every thread calls, the histogram is complete and holds rem or
// more.  out: {bin, above}.
// c0, c1: this thread's counts, of bin b0 and the one below (c1 = 0: it has one),
// the threads' bins falling.
__device__ __forceinline__ void find_bin(int b0, int c0, int c1, int rem, int* red, int* out) {
  const int t = tid(), lane = t & 63, w = t >> 6;
  const int v = wave_scan(c0 + c1);
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  int before = v - c0 - c1;
#pragma unroll
  for (int i = 0; i < kPickWaves; ++i)
    if (i < w) before += red[i];
  if (before < rem && rem <= before + c0 + c1) {
    out[0] = rem <= before + c0 ? b0 : b0 - 1;
    out[1] = rem <= before + c0 ? before : before + c0;
  }
  __syncthreads();
}

// The same for a histogram of 1024 or 2048 bins in LDS.
__device__ __forceinline__ void find_bin(const int* hist, int bins, int rem, int* red, int* out) {
  const int per = bins / kPickThreads, b0 = bins - 1 - per * tid();
  find_bin(b0, hist[b0], per == 2 ? hist[b0 - 1] : 0, rem, red, out);
}

// cnt[0 .. n), n <= 128: exclusive prefix sums in place, their total returned;
// every thread calls.
__device__ __forceinline__ uint32_t scan128(uint32_t* cnt, int n, uint32_t* total) {
  __syncthreads();
  if (tid() < 64) {
    const int i = 2 * tid();
    const uint32_t x0 = i < n ? cnt[i] : 0, x1 = i + 1 < n ? cnt[i + 1] : 0;
    const uint32_t v = wave_scan(x0 + x1);
    if (i < n) cnt[i] = v - x0 - x1;
    if (i + 1 < n) cnt[i + 1] = v - x1;
    if (tid() == 63) *total = v;
  }
  __syncthreads();
  return *total;
}

// One workgroup a unit, which holds the keys of all its rows in registers (TILES x
// 4096 of them): the histogram of each part of the weights that share the parts
// before it leads to the weight of the last row kept; rows of that weight are ranked
// by their order, then holes below the budget and kept rows behind it.  A rank is
// the prefix of per-wave counts (ballots) plus the lanes before.  Bound by latency:
// one read of the rows (8 bytes each), three histograms, two rankings.  Holding eight
// tiles it takes 33 us for 18k to 32k rows, against 190 and 126 with the rows read
// again for every 8 bits and a barrier pair for every 1024 ranked; two tiles are
// where it is even with the launches below.
template <int TILES>
__global__ __launch_bounds__(kPickThreads) void evict_pick(EvictArgs a) {
  __shared__ int hist[kBins];
  __shared__ uint32_t cnt[TILES * kPickWaves];
  __shared__ int red[2 * kPickWaves], out[2];
  __shared__ uint32_t total;
  const int t = tid(), lane = t & 63, w = t >> 6, B = a.budget;
  EvictUnit u;
  if (!evict_unit(a, bid_x(), u)) {
    if (t == 0) a.count[bid_x()] = 0;
    return;
  }
  const int R = u.R;
  if (u.g == 0 && t == 0) a.rows_out[u.slot] = u.left;
  int32_t* kept = a.kept_out ? a.kept_out + (int64_t)u.unit * B : nullptr;
  if (R <= B) {
    if (kept)
      for (int r = t; r < B; r += kPickThreads) kept[r] = kept_in_place(a, u, r);
    if (t == 0) a.count[u.unit] = 0;
    return;
  }
  uint32_t key[TILES][4];
  load_keys<TILES>(a, u, 0, key);
  int sums[2] = {0, 0};  // protected rows, places below B
#pragma unroll
  for (int j = 0; j < TILES; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sums[0] += key[j][e] == kProtected;
      sums[1] += key[j][e] != kAbsent && j * kTileRows + 4 * t + e < B;
    }
  block_sums(sums, red);
  // kept: above T, and of those equal to T the first rem by row
  uint32_t T = kProtected;
  int rem = sums[1];
  if (sums[0] < rem) {
    T = 0;
    rem -= sums[0];
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      const int sh = part_shift(part), bins = part_bins(part);
      for (int i = t; i < bins; i += kPickThreads) hist[i] = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t k = key[j][e];
          const bool same = part == 0 || (k >> part_shift(part ? part - 1 : 0)) == (T >> part_shift(part ? part - 1 : 0));
          if (k != kProtected && k != kAbsent && same) atomicAdd(&hist[(k >> sh) & (bins - 1)], 1);
        }
      __syncthreads();
      find_bin(hist, bins, rem, red, out);
      T |= (uint32_t)out[0] << sh;
      rem -= out[1];
      __syncthreads();
    }
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  // rank the rows of weight T
#pragma unroll
  for (int j = 0; j < TILES; ++j) {
    int c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[j][e] == T));
    if (lane == 0) cnt[j * kPickWaves + w] = c;
  }
  scan128(cnt, TILES * kPickWaves, &total);
  uint32_t keep = 0;  // bit 4 j + e
#pragma unroll
  for (int j = 0; j < TILES; ++j) {
    int before = cnt[j * kPickWaves + w];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(key[j][e] == T) & below);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool eq = key[j][e] == T;
      if (key[j][e] > T || (eq && before < rem)) keep |= 1u << (4 * j + e);
      before += eq;
    }
  }
  // rank the holes below B (low half) and the kept rows from B on (high half)
  __syncthreads();
#pragma unroll
  for (int j = 0; j < TILES; ++j) {
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = j * kTileRows + 4 * t + e;
      const bool k = (keep >> (4 * j + e)) & 1;
      c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(r < B && !k && key[j][e] != kAbsent));
      c += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(r >= B && k)) << 16;
    }
    if (lane == 0) cnt[j * kPickWaves + w] = c;
  }
  const uint32_t all = scan128(cnt, TILES * kPickWaves, &total);
  int32_t* src = a.src + (int64_t)u.unit * a.max_moves;
  int32_t* dst = a.dst + (int64_t)u.unit * a.max_moves;
#pragma unroll
  for (int j = 0; j < TILES; ++j) {
    uint32_t before = cnt[j * kPickWaves + w];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = j * kTileRows + 4 * t + e;
      const bool k = (keep >> (4 * j + e)) & 1;
      before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(r < B && !k && key[j][e] != kAbsent) & below);
      before += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(r >= B && k) & below) << 16;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = j * kTileRows + 4 * t + e;
      const bool k = (keep >> (4 * j + e)) & 1;
      const int hole = before & 0xffff, from = before >> 16;
      if (r < B && key[j][e] == kAbsent) {
        if (kept) kept[r] = -1;
      } else if (r < B && !k) {
        if (debug_check(hole < a.max_moves, kDbgPagedMove)) dst[hole] = r;
        before += 1;
      } else if (r >= B && k) {
        if (debug_check(from < a.max_moves, kDbgPagedMove)) src[from] = r;
        before += 1u << 16;
      } else if (r < B && kept) {
        kept[r] = r;
      }
    }
  }
  if (t == 0) a.count[u.unit] = all & 0xffff;
}

// ---------------------------------------------------------------- selection, split
// The same for more rows than one workgroup takes well, in two launches over about
// 32 splits a unit at most.  The first stores the keys and each split's histogram of
// the leading bits.  In the second every workgroup finds the weight of the last row
// kept by itself: it adds the histograms up, reads the unit's keys for each of the
// other two parts, counts the rows kept before its split, and writes its share of the
// lists.  Nothing is cleared, added atomically in memory or waited for inside a
// launch, and the three reads of 4 bytes a row hit the cache.  1 sequence x 8 heads
// of 32k rows 6.2 + 16.3 us, 8 x 8 of 18k 8.3 + 17.5.
struct SplitArgs {
  uint32_t* keys;  // [units][row_pad]
  int* hist;       // [units][splits][kBins]
  int2* sums;      // [units][splits] protected rows, rows below the budget that are not there
  int64_t row_pad;
  int splits, split_rows;
};

__global__ __launch_bounds__(kPickThreads) void evict_split_keys(EvictArgs a, SplitArgs p) {
  __shared__ int hist[kBins];
  __shared__ int red[2 * kPickWaves];
  const int t = tid(), split = bid_x(), B = a.budget;
  EvictUnit u;
  if (!evict_unit(a, bid_y(), u)) {
    if (t == 0 && split == 0) a.count[bid_y()] = 0;
    return;
  }
  if (u.g == 0 && t == 0 && split == 0) a.rows_out[u.slot] = u.left;
  if (u.R <= B) {
    if (a.kept_out)
      for (int r = split * kPickThreads + t; r < B; r += p.splits * kPickThreads)
        a.kept_out[(int64_t)u.unit * B + r] = kept_in_place(a, u, r);
    if (t == 0 && split == 0) a.count[u.unit] = 0;
    return;
  }
  const int64_t at = (int64_t)u.unit * p.splits + split;
  const int r0 = min((int64_t)split * p.split_rows, (int64_t)u.R), r1 = min((int64_t)r0 + p.split_rows, (int64_t)u.R);
  for (int i = t; i < kBins; i += kPickThreads) hist[i] = 0;
  __syncthreads();
  int sums[2] = {0, 0};
  for (int r = r0; r < r1; r += kTileRows) {
    uint32_t key[1][4];
    load_keys<1>(a, u, r, key);
    const int mine = r + 4 * t;
    if (mine < r1)
      *(u32x4*)(p.keys + (int64_t)u.unit * p.row_pad + mine) = u32x4{key[0][0], key[0][1], key[0][2], key[0][3]};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (mine + e >= r1) break;
      if (key[0][e] == kProtected)
        ++sums[0];
      else if (key[0][e] == kAbsent)
        sums[1] += mine + e < B;
      else
        atomicAdd(&hist[key[0][e] >> part_shift(0)], 1);
    }
  }
  block_sums(sums, red);  // and the histogram is complete
  for (int i = t; i < kBins; i += kPickThreads) p.hist[at * kBins + i] = hist[i];
  if (t == 0) p.sums[at] = make_int2(sums[0], sums[1]);
}

// f(r, keys of rows r .. r + 3) for a unit's stored keys of the rows before `to`,
// four a thread.  (Held in registers between the scans they take as long: a scan is
// bound by its compares.)
template <typename F>
__device__ __forceinline__ void scan_keys(const uint32_t* keys, int to, F f) {
#pragma unroll 4
  for (int r = 4 * tid(); r < to; r += kTileRows) f(r, *(const u32x4*)(keys + r));
}

__global__ __launch_bounds__(kPickThreads) void evict_split_lists(EvictArgs a, SplitArgs p) {
  __shared__ int hist[2][part_bins(1)];
  __shared__ int red[4 * kPickWaves], out[2];
  const int t = tid(), lane = t & 63, w = t >> 6, split = bid_x(), B = a.budget;
  EvictUnit u;
  if (!evict_unit(a, bid_y(), u) || u.R <= B) return;
  const uint32_t* keys = p.keys + (int64_t)u.unit * p.row_pad;
  // the splits' histograms of the leading bits, two bins a thread from the top
  const int* first = p.hist + (int64_t)u.unit * p.splits * kBins + kBins - 2 - 2 * t;
  int2 sums = {0, 0};  // of split `lane` (there are at most 32)
  if (lane < p.splits) sums = p.sums[(int64_t)u.unit * p.splits + lane];
  int c0 = 0, c1 = 0;
#pragma unroll 8
  for (int s = 0; s < p.splits; ++s) {
    const int2 v = *(const int2*)(first + (int64_t)s * kBins);
    c0 += v.y;
    c1 += v.x;
  }
  hist[0][t] = hist[1][t] = 0;
  const int prot = wave_total(sums.x), gone = wave_total(sums.y), gone_before = wave_total(lane < split ? sums.y : 0);
  // kept: above T, and of those equal to T the first rem by row
  uint32_t T = kProtected;
  int rem = B - gone;
  if (prot < rem) {
    rem -= prot;
    find_bin(kBins - 1 - 2 * t, c0, c1, rem, red, out);
    T = (uint32_t)out[0] << part_shift(0);
    rem -= out[1];
#pragma unroll
    for (int part = 1; part < kParts; ++part) {
      __syncthreads();  // out is read
      scan_keys(keys, u.R, [&](int, u32x4 k) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k[e] >> part_shift(part - 1) == T >> part_shift(part - 1))
            atomicAdd(&hist[part - 1][(k[e] >> part_shift(part)) & (part_bins(part) - 1)], 1);
      });
      __syncthreads();
      find_bin(hist[part - 1], part_bins(part), rem, red, out);
      T |= (uint32_t)out[0] << part_shift(part);
      rem -= out[1];
    }
  }
  const int r0 = min((int64_t)split * p.split_rows, (int64_t)u.R), r1 = min((int64_t)r0 + p.split_rows, (int64_t)u.R);
  // rows above T and equal to it before this split, and below B (for the number of
  // moves, and where rows from B on go); rows below B that are not there count as kept
  // where they are
  int c[4] = {0, 0, 0, 0};
  const bool low = split == 0 || r1 > B;
  scan_keys(keys, low ? max(r0, B) : r0, [&](int r, u32x4 k) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[0] += k[e] > T && r + e < r0;
      c[1] += k[e] == T && r + e < r0;
      c[2] += k[e] > T && r + e < B;
      c[3] += k[e] == T && r + e < B;
    }
  });
  block_sums(c, red);
  int eq = c[1], kept_before = c[0] + min(rem, c[1]) + gone_before;
  const int kept_low = c[2] + min(rem, c[3]) + gone;  // low only
  if (t == 0 && split == 0) a.count[u.unit] = B - kept_low;
  int32_t* kept = a.kept_out ? a.kept_out + (int64_t)u.unit * B : nullptr;
  int32_t* src = a.src + (int64_t)u.unit * a.max_moves;
  int32_t* dst = a.dst + (int64_t)u.unit * a.max_moves;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int tile = r0; tile < r1; tile += kTileRows) {
    const int r = tile + 4 * t;
    const u32x4 k = r < r1 ? *(const u32x4*)(keys + r) : u32x4{0u, 0u, 0u, 0u};
    int n = 0, before = eq;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(r + e < r1 && k[e] == T);
      n += __builtin_popcountll(m);
      before += __builtin_popcountll(m & below);
    }
    __syncthreads();
    if (lane == 0) red[w] = n;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPickWaves; ++i) {
      if (i < w) before += red[i];
      eq += red[i];
    }
    bool keep[4];
    int rank = kept_before;  // kept rows before this thread's; the holes before row r are r - rank
    n = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool live = r + e < r1, same = live && k[e] == T;
      keep[e] = live && (k[e] > T || (same && before < rem) || (k[e] == kAbsent && r + e < B));
      before += same;
      const uint64_t m = __builtin_amdgcn_ballot_w64(keep[e]);
      n += __builtin_popcountll(m);
      rank += __builtin_popcountll(m & below);
    }
    __syncthreads();
    if (lane == 0) red[w] = n;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPickWaves; ++i) {
      if (i < w) rank += red[i];
      kept_before += red[i];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (r + e >= r1) break;
      if (r + e < B) {
        if (!keep[e]) {
          if (debug_check(r + e - rank < a.max_moves, kDbgPagedMove)) dst[r + e - rank] = r + e;
        } else if (kept) {
          kept[r + e] = k[e] == kAbsent ? -1 : r + e;
        }
      } else if (keep[e] && debug_check(rank - kept_low < a.max_moves, kDbgPagedMove)) {
        src[rank - kept_low] = r + e;
      }
      rank += keep[e];
    }
  }
}

// block x: share of the moves, y: unit.  8 x 8 units of 1500 moves of 520 bytes (100 MB
// read and written) 23.5 us, 4.2 TB/s; few moves are bound by the chain of dependent
// loads (list, page, row): 8 units of 3700 (31 MB) 9.1 us, 3.4 TB/s.
__global__ __launch_bounds__(256) void evict_move(EvictArgs a, int shares) {
  const int unit = bid_y(), b = unit / a.Hkv, g = unit % a.Hkv;
  const int n = a.count[unit];
  if (n == 0) return;
  const int slot = a.slot_ids[b];
  const int pieces = (a.kbytes + a.vbytes) / 16, kp = a.kbytes / 16;
  const int32_t* src = a.src + (int64_t)unit * a.max_moves;
  const int32_t* dst = a.dst + (int64_t)unit * a.max_moves;
  for (int64_t i = (int64_t)bid_x() * 256 + tid(); i < (int64_t)n * pieces; i += (int64_t)shares * 256) {
    const int j = (int)(i / pieces), c = (int)(i % pieces);
    const int rs = src[j], rd = dst[j];
    if (c == 0 && a.kept_out) a.kept_out[(int64_t)unit * a.budget + rd] = rs;
    const int64_t from = evict_row(a, slot, g, rs), to = evict_row(a, slot, g, rd);
    if (from < 0 || to < 0) continue;  // (the selection names no such row)
    if (c < kp)
      *(u32x4*)(a.ck + to * a.kbytes + 16 * c) = *(const u32x4*)(a.ck + from * a.kbytes + 16 * c);
    else
      *(u32x4*)(a.cv + to * a.vbytes + 16 * (c - kp)) = *(const u32x4*)(a.cv + from * a.vbytes + 16 * (c - kp));
    if (c == 0) {
      a.token[to] = a.token[from];
      a.weight[to] = a.weight[from];
    }
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

SNAP_DEBUG_READER(debug_flags_evict)

EvictGeometry evict_geometry(const snap_params& p, int n, int max_rows) {
  EvictGeometry g{};
  const int units = (n > 0 ? n : 1) * p.n_kv_heads, budget = p.sink + p.recent + p.topk;
  const int behind = max_rows > budget ? max_rows - budget : 0;
  g.max_moves = behind < budget ? behind : budget;
  size_t off = 0;
  g.splits = 0;
  if (max_rows > kPickRows) {
    // a tile each, or more rows where there would be over 32 of them or more
    // workgroups than CUs: every split reads all of its unit's keys
    const int most = units >= 256 ? 1 : (256 / units < 32 ? 256 / units : 32);
    g.split_rows = (int)((max_rows + (int64_t)most * kTileRows - 1) / ((int64_t)most * kTileRows)) * kTileRows;
    g.splits = (max_rows + g.split_rows - 1) / g.split_rows;
    g.row_pad = ((size_t)max_rows + 3) & ~(size_t)3;
    // Room for units * splits histograms, or for more: no call with fewer units or rows
    // has more splits than `room`, so that a workspace of the largest call serves it.
    const int tiles = (int)(((int64_t)max_rows + kTileRows - 1) / kTileRows);
    const size_t each = (size_t)units * (tiles < 32 ? tiles : 32), all = units > 256 ? units : 256;
    const size_t room = each < all ? each : all;
    g.off_keys = off;
    off = align256(off + (size_t)units * g.row_pad * sizeof(uint32_t));
    g.off_hist = off;
    off = align256(off + room * kBins * sizeof(int));
    g.off_sums = off;
    off = align256(off + room * sizeof(int2));
  }
  g.off_count = off;
  off = align256(off + (size_t)units * sizeof(int32_t));
  g.off_src = off;
  off = align256(off + (size_t)units * g.max_moves * sizeof(int32_t));
  g.off_dst = off;
  off = align256(off + (size_t)units * g.max_moves * sizeof(int32_t));
  g.bytes = off;
  return g;
}

snap_status launch_paged_evict(const snap_params& p, const snap_paged_cache& c, const int32_t* rows, const int32_t* pos,
                               int32_t* rows_out, int n, const int32_t* slot_ids, int max_rows, int32_t* kept_out,
                               void* ws, hipStream_t stream) {
  const EvictGeometry geo = evict_geometry(p, n, max_rows);
  const int elt = p.kv_dtype == SNAP_F32 ? 4 : (p.kv_dtype == SNAP_BF16 ? 2 : 1);
  EvictArgs a = {};
  a.ck = (unsigned char*)c.k;
  a.cv = p.v_in_k ? nullptr : (unsigned char*)c.v;
  a.token = c.token;
  a.weight = c.weight;
  a.rows = rows;
  a.pos = pos;
  a.rows_out = rows_out;
  a.slot_ids = slot_ids;
  a.table = c.page_table;
  a.kept_out = kept_out;
  a.count = (int32_t*)((unsigned char*)ws + geo.off_count);
  a.src = (int32_t*)((unsigned char*)ws + geo.off_src);
  a.dst = (int32_t*)((unsigned char*)ws + geo.off_dst);
  a.Hkv = p.n_kv_heads;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = 31 - __builtin_clz((unsigned)c.page_size);
  a.max_pages = c.max_pages;
  a.max_rows = max_rows;
  a.budget = p.sink + p.recent + p.topk;
  a.sink = p.sink;
  a.recent = p.recent;
  a.max_moves = geo.max_moves;
  a.kbytes = p.d_qk * elt;
  a.vbytes = p.v_in_k ? 0 : p.d_v * elt;
  const int units = n * p.n_kv_heads;
  if (!geo.splits) {
    hipLaunchKernelGGL(evict_pick<kPickRows / kTileRows>, dim3(units), dim3(kPickThreads), 0, stream, a);
  } else {
    unsigned char* base = (unsigned char*)ws;
    SplitArgs sp;
    sp.keys = (uint32_t*)(base + geo.off_keys);
    sp.hist = (int*)(base + geo.off_hist);
    sp.sums = (int2*)(base + geo.off_sums);
    sp.row_pad = (int64_t)geo.row_pad;
    sp.splits = geo.splits;
    sp.split_rows = geo.split_rows;
    const dim3 grid(geo.splits, units);
    hipLaunchKernelGGL(evict_split_keys, grid, dim3(kPickThreads), 0, stream, a, sp);
    if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
    hipLaunchKernelGGL(evict_split_lists, grid, dim3(kPickThreads), 0, stream, a, sp);
  }
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  if (geo.max_moves > 0) {
    const int64_t pieces = (int64_t)geo.max_moves * ((a.kbytes + a.vbytes) / 16);
    const int shares = (int)(pieces < 256 * 256 ? (pieces + 255) / 256 : 256);
    hipLaunchKernelGGL(evict_move, dim3(shares, units), dim3(256), 0, stream, a, shares);
    if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  }
  return SNAP_OK;
}

}  // namespace snap
