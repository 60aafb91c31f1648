// pages.hip -- page tables on the device: pages handed out to sequences that grow,
// taken back, and the map of a packed batch's tokens to their rows.
//
//   pages_reserve   one workgroup: what each sequence lacks, served in order by
//                   prefix sums, the pages copied off the end of the free list
//   pages_release   one workgroup: the reverse
//   pages_map       a workgroup for every kMapTokens tokens, each after its own
//                   prefix sums of the lengths
//
// All are bound by latency: a handful of dependent loads, no more than 12 bytes a
// token written.  One token each of 64 sequences 3 us a call; 24 prompts of up to 32k
// tokens (6200 pages of 64) 6.5 us, and about 20 for 48000 pages, by what one CU stores.
#include "lds_dma.h"
#include "snap_internal.h"

namespace snap {

namespace {

constexpr int kPoolThreads = 1024;
constexpr int kPoolWaves = kPoolThreads / 64;
constexpr int kAtOnce = 4;  // pages that a thread has in flight

struct PoolArgs {
  int32_t* table;
  int32_t* held;
  int32_t* free_pages;
  int32_t* n_free;
  const int32_t* rows;
  const int32_t* slot_ids;
  const int32_t* lengths;
  int32_t* short_out;
  int n, len, n_slots, n_pages, page_shift, max_pages;
};

// Inclusive prefix sum of numbers that are not negative over a workgroup of W waves (every
// thread calls); `total`: of all.  64 bits: a thousand sequences may lack 2^24 pages each.
template <int W>
__device__ __forceinline__ int64_t group_scan(int x, int64_t* red, int64_t& total) {
  const int lane = tid() & 63, w = tid() >> 6;
  int64_t v = wave_scan(x & 0xffff) + ((int64_t)wave_scan(x >> 16) << 16);
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (i < w) v += red[i];
    total += red[i];
  }
  return v;
}

// The last i in [0, 1 << BITS) with at[i] <= x (at[0] <= x, at does not fall).
template <int BITS>
__device__ __forceinline__ int find_last(const int* at, int x) {
  int i = 0;
#pragma unroll
  for (int s = 1 << (BITS - 1); s; s >>= 1)
    if (at[i + s] <= x) i += s;
  return i;
}

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Whether the workgroup's threads name a slot (>= 0) twice, by a table of open addresses in
// LDS (all its entries -1 before, at a barrier).
constexpr int kSeen = 2 * kPoolThreads;
__device__ __forceinline__ void note_slot(int* seen, int* twice, int slot) {
  if (slot < 0) return;
  uint32_t at = ((uint32_t)slot * 2654435761u) >> 21;  // (half full at most: a free entry is met)
  for (;; at = (at + 1) & (kSeen - 1)) {
    const int was = atomicCAS(&seen[at], -1, slot);
    if (was == -1) return;
    if (was == slot) {
      *twice = 1;
      return;
    }
  }
}

// Sequence t of a chunk is thread t.  Where all sequences of the chunk before it fit,
// so do their pages' ranks: page e of the chunk is rank e of those taken.
// A slot named again: pages are handed out up to some sequence and to none behind it.  Up
// to there all earlier wishes of the slot were granted, so that the sequence lacks what its
// own exceeds the largest of them by; behind it is served only if the slot holds enough.
// (A search of the chunk for each sequence, where a slot is named twice.)
__global__ __launch_bounds__(kPoolThreads) void pages_reserve(PoolArgs a) {
  __shared__ int64_t red[kPoolWaves];
  __shared__ int first[kPoolThreads], to[kPoolThreads];  // rank of a sequence's first page, its table entry less that rank
  __shared__ int slots[kPoolThreads], wants[kPoolThreads], seen[kSeen], twice;
  const int t = tid();
  const int free0 = clamp_int(*a.n_free, 0, a.n_pages);
  int64_t before = 0;  // pages lacked by the chunks before
  int taken = 0;
  for (int b0 = 0; b0 < a.n; b0 += kPoolThreads) {
    const int b = b0 + t;
    int slot = b < a.n ? a.slot_ids[b] : -1;
    const int add = b < a.n ? (a.lengths ? a.lengths[b] : a.len) : 0;
    for (int i = t; i < kSeen; i += kPoolThreads) seen[i] = -1;
    if (t == 0) twice = 0;
    if (slot < 0 || slot >= a.n_slots) slot = -1;
    const int r = slot >= 0 ? a.rows[slot] : -1, held = slot >= 0 ? a.held[slot] : 0;
    lds_barrier();  // (the loads stay in flight)
    note_slot(seen, &twice, slot);
    const int h0 = clamp_int(held, 0, a.max_pages);
    const int64_t want = ((int64_t)(r < 0 ? 0 : r) + (add < 0 ? 0 : add) + (1 << a.page_shift) - 1) >> a.page_shift;
    const bool fits = want <= a.max_pages, live = slot >= 0 && r >= 0;
    slots[t] = slot;
    wants[t] = live && fits ? (int)want : 0;
    lds_barrier();
    const bool again = twice != 0;
    // the most of the wishes of this slot, before this one or of all, and what the slot holds
    auto most = [&](int upto) {
      int h = h0;
      for (int i = 0; i < upto; ++i)
        if (slots[i] == slot) h = max(h, wants[i]);
      return h;
    };
    int h = again && live ? most(t) : h0;
    int64_t lack = live && want > h ? want - h : 0;
    int64_t total;
    const int64_t upto = before + group_scan<kPoolWaves>(fits ? (int)lack : 0, red, total);
    bool served = fits && (lack == 0 || upto <= free0), last = true;
    const int take = served ? (int)lack : 0;
    int64_t chunk;
    const int rank = (int)group_scan<kPoolWaves>(take, red, chunk) - take;
    if (again) {  // by the wishes that were granted
      wants[t] = take ? (int)want : 0;
      __syncthreads();
      if (live) {
        h = most(t);
        lack = want > h ? want - h : 0;
        served = fits && (take || lack == 0);
        last = take && (int)want == most(kPoolThreads);
      }
    }
    if (b < a.n && a.short_out) a.short_out[b] = served ? 0 : (int)(lack < 0x7fffffff ? lack : 0x7fffffff);
    if (take && last) a.held[slot] = (int)want;
    first[t] = rank;
    to[t] = h - rank;
    __syncthreads();
    for (int e0 = t; e0 < (int)chunk; e0 += kAtOnce * kPoolThreads) {
      int page[kAtOnce], s[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) page[i] = a.free_pages[free0 - 1 - taken - min(e0 + i * kPoolThreads, (int)chunk - 1)];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) s[i] = find_last<10>(first, e0 + i * kPoolThreads);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (e0 + i * kPoolThreads < (int)chunk)
          a.table[(size_t)slots[s[i]] * a.max_pages + to[s[i]] + e0 + i * kPoolThreads] = page[i];
    }
    taken += (int)chunk;
    before += total;
    __syncthreads();
  }
  if (t == 0) *a.n_free = free0 - taken;
}

// Chunks of sequences from the last to the first, each chunk's pages in reverse: the
// order in which pages_reserve would take them again.
__global__ __launch_bounds__(kPoolThreads) void pages_release(PoolArgs a) {
  __shared__ int64_t red[kPoolWaves];
  __shared__ int first[kPoolThreads], from[kPoolThreads], slots[kPoolThreads], seen[kSeen], twice;
  const int t = tid();
  int64_t end = clamp_int(*a.n_free, 0, a.n_pages);
  for (int b0 = (a.n - 1) / kPoolThreads * kPoolThreads; b0 >= 0; b0 -= kPoolThreads) {
    const int b = b0 + t;
    int slot = b < a.n ? a.slot_ids[b] : -1;
    if (slot < 0 || slot >= a.n_slots) slot = -1;
    for (int i = t; i < kSeen; i += kPoolThreads) seen[i] = -1;
    if (t == 0) twice = 0;
    slots[t] = slot;
    const int r = slot >= 0 ? a.rows[slot] : 0, held = slot >= 0 ? a.held[slot] : 0;
    lds_barrier();  // (the loads stay in flight)
    note_slot(seen, &twice, slot);
    const int h = clamp_int(held, 0, a.max_pages);
    lds_barrier();
    const int keep = min((int)(((int64_t)(r < 0 ? 0 : r) + (1 << a.page_shift) - 1) >> a.page_shift), h);
    int give = h - keep;
    if (twice)  // (the last of those that name the slot)
      for (int i = t + 1; i < kPoolThreads; ++i)
        if (slots[i] == slot) give = 0;
    int64_t all, chunk;
    // more than there are pages would be entries that were handed back twice: left out
    if (end + group_scan<kPoolWaves>(give, red, all) > a.n_pages) give = 0;
    const int rank = (int)group_scan<kPoolWaves>(give, red, chunk) - give, m = (int)chunk;
    if (give) a.held[slot] = keep;
    first[t] = rank;
    from[t] = keep - rank;
    __syncthreads();
    for (int e0 = t; e0 < m; e0 += kAtOnce * kPoolThreads) {
      int32_t* at[kAtOnce];
      int page[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int e = min(e0 + i * kPoolThreads, m - 1), s = find_last<10>(first, e);
        at[i] = a.table + (size_t)slots[s] * a.max_pages + from[s] + e;
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) page[i] = *at[i];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (e0 + i * kPoolThreads < m) {
          a.free_pages[end + m - 1 - (e0 + i * kPoolThreads)] = page[i];
          *at[i] = -1;
        }
    }
    end += m;
    __syncthreads();
  }
  if (t == 0) *a.n_free = (int)end;
}

constexpr int kMapThreads = 256, kMapTokens = 1024;

struct MapArgs {
  const int32_t* table;
  const int32_t* rows;
  const int32_t* pos;
  const int32_t* slot_ids;
  const int32_t* lengths;
  int32_t* starts;
  int32_t* seq_of;
  int32_t* row_of;
  int32_t* pos_of;
  int n, tokens, n_slots, n_pages, page_shift, max_pages;
};

__global__ __launch_bounds__(kMapThreads) void pages_map(MapArgs a) {
  __shared__ int64_t red[kMapThreads / 64];
  __shared__ int first[kMapThreads], slots[kMapThreads], rows[kMapThreads], pos[kMapThreads];
  const int t = tid(), lo = bid_x() * kMapTokens;
  const int hi = a.tokens - lo < kMapTokens ? a.tokens : lo + kMapTokens;
  int64_t before = 0;
  for (int b0 = 0; b0 < a.n; b0 += kMapThreads) {
    const int b = b0 + t;
    int len = b < a.n ? a.lengths[b] : 0, slot = b < a.n ? a.slot_ids[b] : -1;
    len = len < 0 ? 0 : len;
    if (slot < 0 || slot >= a.n_slots) slot = -1;
    const int r = slot >= 0 ? a.rows[slot] : -1;
    int64_t total;
    const int64_t start = before + group_scan<kMapThreads / 64>(len, red, total) - len;
    first[t] = start < a.tokens ? (int)start : a.tokens;
    slots[t] = r < 0 ? -1 : slot;
    rows[t] = r;
    pos[t] = r < 0 ? 0 : (a.pos ? a.pos[slot] : r);
    if (bid_x() == 0 && b < a.n) a.starts[b] = first[t];
    __syncthreads();
    const int64_t c1 = before + total;
    for (int i = (before > lo ? (before < hi ? (int)before : hi) : lo) + t; i < (c1 < hi ? c1 : hi); i += kMapThreads) {
      const int s = find_last<8>(first, i), at = i - first[s];
      int64_t row = -1;
      if (slots[s] >= 0) {
        const int64_t x = (int64_t)rows[s] + at, p = x >> a.page_shift;
        const int page = p < a.max_pages ? a.table[(size_t)slots[s] * a.max_pages + p] : -1;
        if (page >= 0 && page < a.n_pages) row = ((int64_t)page << a.page_shift) + (x & ((1 << a.page_shift) - 1));
      }
      a.seq_of[i] = b0 + s;
      a.row_of[i] = (int)row;
      a.pos_of[i] = slots[s] >= 0 ? (int)((uint32_t)pos[s] + (uint32_t)at) : 0;
    }
    before = c1;
    __syncthreads();
    if (bid_x() != 0 && before >= hi) return;  // (the first workgroup has every start to write)
  }
  for (int i = (before > lo ? (before < hi ? (int)before : hi) : lo) + t; i < hi; i += kMapThreads) {
    a.seq_of[i] = -1;
    a.row_of[i] = -1;
    a.pos_of[i] = 0;
  }
  if (bid_x() == 0 && t == 0) a.starts[a.n] = before < a.tokens ? (int)before : a.tokens;
}

inline int log2_of(int x) { return 31 - __builtin_clz((unsigned)x); }

PoolArgs pool_args(const snap_page_pool& c, const int32_t* rows, int n, const int32_t* slot_ids) {
  PoolArgs a = {};
  a.table = c.page_table;
  a.held = c.held;
  a.free_pages = c.free_pages;
  a.n_free = c.n_free;
  a.rows = rows;
  a.slot_ids = slot_ids;
  a.n = n;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = log2_of(c.page_size);
  a.max_pages = c.max_pages;
  return a;
}

}  // namespace

snap_status launch_pages_reserve(const snap_page_pool& c, const int32_t* rows, int n, const int32_t* slot_ids,
                                 const int32_t* lengths, int len, int32_t* short_out, hipStream_t stream) {
  PoolArgs a = pool_args(c, rows, n, slot_ids);
  a.lengths = lengths;
  a.len = len;
  a.short_out = short_out;
  hipLaunchKernelGGL(pages_reserve, dim3(1), dim3(kPoolThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

snap_status launch_pages_release(const snap_page_pool& c, const int32_t* rows, int n, const int32_t* slot_ids,
                                 hipStream_t stream) {
  const PoolArgs a = pool_args(c, rows, n, slot_ids);
  hipLaunchKernelGGL(pages_release, dim3(1), dim3(kPoolThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

snap_status launch_pages_map(const snap_page_pool& c, const int32_t* rows, const int32_t* pos, int n,
                             const int32_t* slot_ids, const int32_t* lengths, int tokens, int32_t* starts,
                             int32_t* seq_of, int32_t* row_of, int32_t* pos_of, hipStream_t stream) {
  MapArgs a = {};
  a.table = c.page_table;
  a.rows = rows;
  a.pos = pos;
  a.slot_ids = slot_ids;
  a.lengths = lengths;
  a.starts = starts;
  a.seq_of = seq_of;
  a.row_of = row_of;
  a.pos_of = pos_of;
  a.n = n;
  a.tokens = tokens;
  a.n_slots = c.n_slots;
  a.n_pages = c.n_pages;
  a.page_shift = log2_of(c.page_size);
  a.max_pages = c.max_pages;
  const int groups = tokens > 0 ? (int)(((int64_t)tokens + kMapTokens - 1) / kMapTokens) : 1;
  hipLaunchKernelGGL(pages_map, dim3(groups), dim3(kMapThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SNAP_OK : SNAP_ERR_HIP;
}

}  // namespace snap
