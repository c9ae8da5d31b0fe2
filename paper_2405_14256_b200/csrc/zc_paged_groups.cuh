// Groups of requests that begin alike: what the kernel of the shared keys and that of the requests' own keys both work out
// from the lengths, each for itself, before they run side by side.
#pragma once
#include "zc_paged_tc.cuh"

namespace {

constexpr int kMaxGroups = ZC_PAGED_MAX_GROUPS;
constexpr int kShareStep = 16;      // shared keys are taken in whole blocks of the own keys' kernel
constexpr int kShareTile = 64;      // keys of a tile of the chunk kernel
// Keys that are not read again, from which on a group is one: an item costs about 25 * 220 cycles beside its tiles, the
// own keys' kernel 20 cycles a key and request.  And of all groups and KV heads together, from which on any is: the shared
// keys' kernel takes some 10 us however few they are, in which 50 MB are read.
constexpr int kWorthSharing = 512;
constexpr long long kWorthAll = 100000;
// Costs as measured, in 220 cycles: a tile of a wide item (both groups of warps work on it), of a narrow one (they take
// turns), an item beside its tiles (Q, first product, output, masks); of the own keys' kernel 128 keys, and a
// (request, KV head) beside them.
constexpr int kWideTile = 7, kNarrowTile = 5, kItemCost = 25;
constexpr int kOwnStep = 4, kOwnUnit = 2;
constexpr int kPlanReq = 768;       // requests whose lengths are kept in shared memory; those of more are read again

// Warps of the own keys' kernel on an SM.
constexpr int kOwnWarps = 8;

// What is known of the groups and the requests, in shared memory.
struct GroupTables {
  int *border, *row;          // [n + 1] first request of a group, its first row
  int *keys, *count, *lead;   // [n] keys that it shares (0: none), its requests that have rows, the first of these
  int *first, *kv;            // [n_req + 1], [n_req] a request's first row, its tokens (n_req <= kPlanReq)
  long long* sums;            // [4] costs of the shared and of the own keys, items of a KV head, keys spared
  int n;
  bool held;
  static constexpr int kInts = 5 * kMaxGroups + 8 + 2 * kPlanReq + 3;   // (8 of them the sums)
  __device__ __forceinline__ GroupTables(void* at, int n_groups, int n_req) {
    sums = reinterpret_cast<long long*>(at);
    border = reinterpret_cast<int*>(sums + 4);
    row = border + kMaxGroups + 1;
    keys = row + kMaxGroups + 1;
    count = keys + kMaxGroups;
    lead = count + kMaxGroups;
    first = lead + kMaxGroups;
    kv = first + kPlanReq + 1;
    n = n_groups;
    held = n_req <= kPlanReq;
  }
  __device__ __forceinline__ int group_of(int r) const {   // -1: none
    if (r < border[0] || r >= border[n]) return -1;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (border[m] <= r) lo = m; else hi = m;
    }
    return lo;
  }
  // The first of a group's requests that has rows (a third atomic beside the minimum and the count would take 1.6 us): the
  // last one that begins where the group's rows do.
  __device__ __forceinline__ int lead_of(const ZcPagedArgs& a, int g) const {
    auto row_of = [&](int r) { return held ? first[r] : min(max(a.row_start[r], 0), a.n_rows); };
    int lo = border[g], hi = border[g + 1];
    if (row_of(lo + 1) > row[g]) return lo;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (row_of(m) <= row[g]) lo = m; else hi = m;
    }
    return lo;
  }
  __device__ __forceinline__ int keys_of(int r) const {
    const int g = group_of(r);
    return g < 0 ? 0 : keys[g];
  }
  __device__ __forceinline__ Chunk chunk(const ZcPagedArgs& a, int r) const {   // load_chunk's
    if (!held) return load_chunk(a, r);
    const int e0 = first[r], e1 = max(first[r + 1], e0);
    Chunk c;
    c.row0 = e0;
    c.n = min(e1 - e0, a.max_rows);
    c.p0 = kv[r] - (e1 - e0);
    return c;
  }
};
__device__ __forceinline__ int group_border(const ZcPagedArgs& a, const ZcGroups& gr, int g) {
  return min(max(gr.start[g], 0), a.n_req);
}

// *sum += v of all threads of the block's warps (64-bit additions in shared memory retry until nobody else is at it: one to
// a warp; one to a thread took 4 us of 64 threads, 10 of 128).
__device__ __forceinline__ void add_all(long long* sum, long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0 && v) atomicAdd(reinterpret_cast<unsigned long long*>(sum), (unsigned long long)v);
}

// How many keys each group shares: at most what the caller says and what lies before every row of its requests, in whole
// blocks of 16 (the keys behind them are the requests' own, as far as this call goes); none where that does not pay.
// Returns how many of the n_cta CTAs that share the GPU are the shared keys' (0: there are none): as many as their cost is
// of all.
template <int THREADS>
__device__ __forceinline__ int plan_groups(const ZcPagedArgs& a, const ZcGroups& gr, const GroupTables& t, int tpt, int n_cta) {
  const int tid = threadIdx.x, n = t.n;
  const long long cap = (long long)a.table_width << a.page_log2;
  // (everything that is read, in one round trip)
  for (int g = tid; g <= n; g += THREADS) {
    t.border[g] = group_border(a, gr, g);
    if (g < n) {
      t.keys[g] = (int)min((long long)max(gr.shared[g], 0), cap);
      t.count[g] = 0;
    }
  }
  if (t.held)
    for (int r = tid; r <= a.n_req; r += THREADS) {
      t.first[r] = min(max(a.row_start[r], 0), a.n_rows);
      if (r < a.n_req) t.kv[r] = (int)min((long long)max(a.kv_len[r], 0), cap);
    }
  if (tid < 4) t.sums[tid] = 0;
  __syncthreads();
  for (int g = tid; g <= n; g += THREADS)
    t.row[g] = t.held ? t.first[t.border[g]] : min(max(a.row_start[t.border[g]], 0), a.n_rows);
  for (int r0 = 0; r0 < a.n_req; r0 += THREADS) {
    const int r = r0 + tid;
    Chunk c;
    c.n = c.p0 = 0;
    if (r < a.n_req) c = t.chunk(a, r);
    const int g = c.n > 0 ? t.group_of(r) : -1;
    // (a warp's requests are one group's as a rule: one of its threads speaks for all)
    const int top = __reduce_max_sync(0xffffffffu, g);
    if (__all_sync(0xffffffffu, g == top || g < 0)) {
      const int least = __reduce_min_sync(0xffffffffu, g < 0 ? 0x7fffffff : c.p0);
      const int count = __popc(__ballot_sync(0xffffffffu, g >= 0));
      if (top >= 0 && (tid & 31) == 0) {
        atomicMin(&t.keys[top], least);
        atomicAdd(&t.count[top], count);
      }
    } else if (g >= 0) {
      atomicMin(&t.keys[g], c.p0);
      atomicAdd(&t.count[g], 1);
    }
  }
  __syncthreads();
  long long cost = 0, items = 0, spared = 0;
  for (int g = tid; g < n; g += THREADS) {
    const int keys = max(t.keys[g], 0) & -kShareStep, rows = t.row[g + 1] - t.row[g], tpi = 2 * tpt;
    const long long mine = (long long)(t.count[g] - 1) * keys;
    const bool on = rows > 0 && n_cta > 1 && mine >= kWorthSharing;
    t.keys[g] = on ? keys : 0;
    if (!on) continue;
    t.lead[g] = t.lead_of(a, g);
    spared += mine;
    const int tiles = (keys + kShareTile - 1) / kShareTile, whole = rows / tpi, rest = rows - whole * tpi;
    cost += (long long)whole * (tiles * kWideTile + kItemCost);
    items += whole + (rest > 0);
    if (rest) cost += tiles * (rest <= tpt ? kNarrowTile : kWideTile) + kItemCost;
  }
  add_all(&t.sums[0], cost);
  add_all(&t.sums[2], items);
  add_all(&t.sums[3], spared);
  __syncthreads();
  if (t.sums[3] * a.h_kv < kWorthAll) {
    for (int g = tid; g < n; g += THREADS) t.keys[g] = 0;
    if (tid == 0) t.sums[0] = 0;
    __syncthreads();
  }
  long long own = 0;
  for (int r = tid; r < a.n_req; r += THREADS) {
    const Chunk c = t.chunk(a, r);
    if (c.n <= 0) continue;
    const int keys = c.p0 + c.n - t.keys_of(r);
    own += (long long)max(1, (keys + 127) >> 7) * kOwnStep + kOwnUnit;
  }
  add_all(&t.sums[1], own);
  __syncthreads();
  const long long shared = t.sums[0], all = shared + t.sums[1];
  if (shared == 0) return 0;
  // (to 24 bits, so that the quotient is one of 32)
  const int shift = max(0, 40 - __clzll(all));
  const uint32_t x = (uint32_t)(shared >> shift), y = (uint32_t)(all >> shift);
  uint32_t mine = min((uint32_t)n_cta - 1u, max(1u, ((uint32_t)n_cta * x + y / 2) / y));
  // As many for each item, where there are more CTAs than items: a share that straddles two items has both their ends.
  // Of the two numbers next to an equal one, that which ends sooner: rounded, 16 items on 148 SMs went from 6 CTAs each to
  // 7, and the own keys of 128 requests from 52 SMs to 36 (95 -> 142 us).  And no more than 2 sqrt(tiles of an item),
  // beyond 8: a piece more takes the joining kernel a quarter as long as a tile.
  const long long all_items = t.sums[2] * a.h_kv;
  if (all_items <= mine) {
    const uint32_t n = (uint32_t)all_items, tiles = (uint32_t)min(1LL << 24, t.sums[0] / t.sums[2]) / kWideTile;
    uint32_t each = mine / n;
    const long long left = (long long)n_cta - n * (each + 1);
    if (left > 0 && x * left > (long long)(y - x) * (n * each)) ++each;
    while (each > 8 && each * each > 4 * tiles) --each;
    mine = n * each;
  }
  return (int)mine;
}

}  // namespace
