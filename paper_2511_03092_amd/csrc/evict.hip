// evict.hip -- eviction from the paged cache by accumulated attention weight.
//
//   evict_select  one workgroup per (sequence, KV head): the weight of the last
//                 row kept (radix select over the weights' bits), then the rows
//                 to move and where to, in ascending order of both
//   evict_move    copies those rows; sources lie from the budget on and
//                 destinations below it, so no row is both
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

// A row's rank among those that are not protected: its weight's bits (weights
// are not negative, so their bits are in their order; NaN and negative: 0).
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w);
  return u > 0x7f800000u ? 0u : u;
}

constexpr int kSelThreads1 = 1024;
constexpr int kSelWaves = kSelThreads1 / 64;

// The number of threads before this one for which pred holds, and of all
// (every thread calls; red: one int per wave).
__device__ __forceinline__ int block_rank(bool pred, int* red, int& all) {
  const int lane = tid() & 63, w = tid() >> 6;
  const uint64_t m = __builtin_amdgcn_ballot_w64(pred);
  __syncthreads();
  if (lane == 0) red[w] = __builtin_popcountll(m);
  __syncthreads();
  int before = 0;
  all = 0;
  for (int i = 0; i < kSelWaves; ++i) {
    if (i < w) before += red[i];
    all += red[i];
  }
  return before + __builtin_popcountll(m & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kSelThreads1) void evict_select(EvictArgs a) {
  __shared__ int hist[256];
  __shared__ int red[kSelWaves];
  __shared__ int pick[2];
  const int unit = bid_x(), b = unit / a.Hkv, g = unit % a.Hkv, t = tid();
  const int slot = a.slot_ids[b], B = a.budget;
  if (slot < 0 || slot >= a.n_slots) {
    if (t == 0) a.count[unit] = 0;
    return;
  }
  int R = a.rows[slot];
  R = R < 0 ? 0 : (R > a.max_rows ? a.max_rows : R);
  if (g == 0 && t == 0) a.rows_out[slot] = R < B ? R : B;
  int32_t* kept = a.kept_out ? a.kept_out + (int64_t)unit * B : nullptr;
  if (R <= B) {
    if (kept)
      for (int r = t; r < B; r += kSelThreads1) kept[r] = r < R ? r : -1;
    if (t == 0) a.count[unit] = 0;
    return;
  }
  const int late = a.pos[slot] - a.recent;
  // state of row r: protected, or its key
  auto look = [&](int r, uint32_t& key) {
    key = 0;
    if (r >= R) return false;
    const int64_t row = evict_row(a, slot, g, r);
    if (row < 0) return false;
    const int tok = a.token[row];
    key = weight_key(a.weight[row]);
    return tok < a.sink || tok >= late;
  };
  int prot = 0;
  for (int r0 = 0; r0 < R; r0 += kSelThreads1) {
    uint32_t key;
    int all;
    block_rank(look(r0 + t, key), red, all);
    prot += all;
  }
  int want = B - prot;  // others that are kept
  uint32_t prefix = 0, known = 0;
  int rem = want;  // kept among those that share the prefix
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (t < 256) hist[t] = 0;
      __syncthreads();
      for (int r = t; r < R; r += kSelThreads1) {
        uint32_t key;
        if (!look(r, key) && (key & known) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
      }
      __syncthreads();
      if (t == 0) {
        int above = 0, d = 255;
        while (d > 0 && above + hist[d] < rem) above += hist[d--];
        pick[0] = d;
        pick[1] = above;
      }
      __syncthreads();
      prefix |= (uint32_t)pick[0] << shift;
      known |= 255u << shift;
      rem -= pick[1];
    }
  }
  // rem rows of weight `prefix` are kept, the lower ones
  int n_prot = 0, n_eq = 0, n_src = 0, n_hole = 0;
  int32_t* src = a.src + (int64_t)unit * a.max_moves;
  int32_t* dst = a.dst + (int64_t)unit * a.max_moves;
  for (int r0 = 0; r0 < R; r0 += kSelThreads1) {
    const int r = r0 + t;
    uint32_t key;
    int all;
    const bool p = look(r, key);
    const int prot_before = n_prot + block_rank(p, red, all);
    n_prot += all;
    bool keep = p && prot_before < B;
    const bool eq = want > 0 && r < R && !p && key == prefix;
    const int eq_before = n_eq + block_rank(eq, red, all);
    n_eq += all;
    keep = keep || (want > 0 && r < R && !p && key > prefix) || (eq && eq_before < rem);
    const bool hole = r < B && !keep, from = r >= B && keep;
    const int at_hole = n_hole + block_rank(hole, red, all);
    n_hole += all;
    const int at_src = n_src + block_rank(from, red, all);
    n_src += all;
    if (hole && debug_check(at_hole < a.max_moves, kDbgPagedMove)) dst[at_hole] = r;
    if (from && debug_check(at_src < a.max_moves, kDbgPagedMove)) src[at_src] = r;
    if (kept && r < B && keep) kept[r] = r;
  }
  if (t == 0) a.count[unit] = n_src < n_hole ? n_src : n_hole;
}

// block x: share of the moves, y: unit
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
    if (from < 0 || to < 0) continue;
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
  hipLaunchKernelGGL(evict_select, dim3(units), dim3(kSelThreads1), 0, stream, a);
  if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  if (geo.max_moves > 0) {
    const int64_t pieces = (int64_t)geo.max_moves * ((a.kbytes + a.vbytes) / 16);
    const int shares = (int)(pieces < 256 * 64 ? (pieces + 255) / 256 : 64);
    hipLaunchKernelGGL(evict_move, dim3(shares, units), dim3(256), 0, stream, a, shares);
    if (hipGetLastError() != hipSuccess) return SNAP_ERR_HIP;
  }
  return SNAP_OK;
}

}  // namespace snap
