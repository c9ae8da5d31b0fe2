// What makes room in the pages: the selection of the tokens that a request keeps, by the weight that attention has
// given them (zc_page_select), and the compaction of their rows to the front of the request's pages (zc_page_compact).
#include "zc_paged.cuh"

namespace {

__device__ __forceinline__ int clamp_len(int n, int width, int page_log2) {
  const long long cap = (long long)width << page_log2;
  return (int)min((long long)max(n, 0), cap);
}

// ---------------------------------------------------------------- selection
// One CTA per (request, KV head).  The candidates' scores become whole numbers of the same order and stay in shared
// memory (as many as there is room for; the rest is fetched again where it is needed), four consecutive ones a thread.
// The k-th highest is found digit by digit (11, 11 and 10 bits) in a histogram of 2048 places; then every thread counts its
// own stretch of positions, and writes the kept ones behind those of the threads before it, so that the list ascends.  Of
// the candidates equal to the k-th the first ones are kept.  Candidates of the first digit found, where they are few, go
// to a list that the other two digits are found in.
// Bound: issue slots (60 %) and the candidates that there is no room for: 64 requests of 8192-16384 tokens, 8 KV heads, 35 us,
// 28 if none were fetched again; reading them from HBM takes 5.  4 requests of 300-512: 4.6 us, a launch and round trips.
// (A word of marks for every 32 positions, set once and resolved from the list: 30 us, and 5.9 for the small ones.)
constexpr int kBins = 2048;
constexpr int kListMost = 1024;
constexpr int kSelectRoom = 226 * 1024, kSelectFixed = 14 * 1024;   // an SM's shared memory; a CTA's beside the keys

// A whole number in the scores' order: NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  const uint32_t k = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return (u << 1) > 0xff000000u ? 0u : k;
}

// Exclusive sums of a and b over the block's threads; returns the whole sums.
template <int THREADS>
__device__ __forceinline__ int2 block_before(int& a, int& b, int2* s_warp) {
  constexpr int kWarps = THREADS / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = a, y = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) {
      x += u;
      y += v;
    }
  }
  if (lane == 31) s_warp[warp] = make_int2(x, y);
  __syncthreads();
  // (every warp sums the warps before it)
  const int2 w = lane < kWarps ? s_warp[lane] : make_int2(0, 0);
  a = x - a + __reduce_add_sync(0xffffffffu, lane < warp ? w.x : 0);
  b = y - b + __reduce_add_sync(0xffffffffu, lane < warp ? w.y : 0);
  return make_int2(__reduce_add_sync(0xffffffffu, w.x), __reduce_add_sync(0xffffffffu, w.y));
}

struct SelectArgs {
  const int32_t *table, *kv_len, *keep, *first;
  const float* scores;
  int32_t *kept, *kept_len;
  int width, page_log2, n_pages, h_kv, recent, max_keep, held;   // held: fours that shared memory has room for
};

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 2048 / THREADS) k_page_select(const SelectArgs a) {
  constexpr int kWarps = THREADS / 32, kPer = kBins / THREADS;
  extern __shared__ uint4 s_keys[];
  __shared__ int s_hist[kBins];
  __shared__ uint32_t s_list[kListMost];
  __shared__ int2 s_warp[kWarps];
  __shared__ int s_digit, s_left, s_in, s_listed;
  const int tid = threadIdx.x;
  const int r = blockIdx.x / a.h_kv, head = blockIdx.x - r * a.h_kv;
  zc_let_next_start();
  for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
  zc_wait_for_last();
  const int n = clamp_len(a.kv_len[r], a.width, a.page_log2);
  const int first = a.first ? min(max(a.first[r], 0), n) : 0;
  const int recent = min(a.recent, n - first);
  const int budget = max(min(max(a.keep[r], 0), a.max_keep), first + recent);
  const bool whole = a.keep[r] >= n || budget >= n || budget > a.max_keep;   // nothing is evicted
  const int len = whole ? n : budget;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.max_keep;
  if (head == 0 && tid == 0) a.kept_len[r] = len;
  for (int i = min(len, a.max_keep) + tid; i < a.max_keep; i += THREADS) kept[i] = -1;
  if (whole) {
    for (int i = tid; i < min(n, a.max_keep); i += THREADS) kept[i] = i;
    return;
  }
  for (int i = tid; i < first; i += THREADS) kept[i] = i;
  for (int i = tid; i < recent; i += THREADS) kept[len - recent + i] = n - recent + i;
  const int c0 = first, c1 = n - recent;           // candidates: positions c0 .. c1 - 1
  int want = budget - first - recent;              // of which so many stay, fewer than there are
  if (want == 0) return;
  const int32_t* table = a.table + (long long)r * a.width;
  const int mask = (1 << a.page_log2) - 1;
  const uint32_t page_bytes = 4u << a.page_log2;
  const int q0 = c0 >> 2, q1 = (c1 + 3) >> 2;      // in fours, which lie on one page
  auto fetch = [&](int q) {
    const int t = 4 * q, page = table[t >> a.page_log2];
    if (page < 0 || page >= a.n_pages) return make_uint4(0u, 0u, 0u, 0u);
    // (h_kv scores to a token: the numbers of all (page, head) stay in 32 bits)
    const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const char*>(a.scores) +
                                                      (uint64_t)((uint32_t)page * (uint32_t)a.h_kv + head) * page_bytes +
                                                      4u * (t & mask));
    const uint4 u = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
    if (max(max(u.x, u.y), max(u.z, u.w)) <= 0x7f800000u)      // as sums of weights are: no sign, no NaN
      return make_uint4(u.x | 0x80000000u, u.y | 0x80000000u, u.z | 0x80000000u, u.w | 0x80000000u);
    return make_uint4(score_key(v.x), score_key(v.y), score_key(v.z), score_key(v.w));
  };
  // which of a four are candidates (all, but at the ends)
  auto members = [&](int q) {
    unsigned in = 15u;
    if (q == q0) in &= 15u << (c0 - 4 * q);
    if (q == q1 - 1) in &= 15u >> (4 * q1 - c1);
    return in;
  };
  auto keys = [&](int q) { return q - q0 < a.held ? s_keys[q - q0] : fetch(q); };
  // ---- the want-th highest key ----
  __syncthreads();
  for (int qa = q0; qa < q1; qa += 2 * THREADS) {
    uint4 k[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int q = qa + u * THREADS + tid;
      if (q < q1) k[u] = fetch(q);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int q = qa + u * THREADS + tid;
      if (q >= q1) continue;
      if (q - q0 < a.held) s_keys[q - q0] = k[u];
      const unsigned in = members(q);
      const uint32_t bin[4] = {k[u].x >> 21, k[u].y >> 21, k[u].z >> 21, k[u].w >> 21};
      if (in == 15u && bin[0] == bin[1] && bin[0] == bin[2] && bin[0] == bin[3]) {
        atomicAdd(&s_hist[bin[0]], 4);               // (tokens that have no weight yet, say)
        continue;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((in >> j) & 1u) atomicAdd(&s_hist[bin[j]], 1);
    }
  }
  uint32_t found = 0;
  int shift = 21, listed = 0;
#pragma unroll 1
  for (int pass = 0;; ++pass) {
    __syncthreads();
    // places from the top: thread t has the kPer places below those of thread t - 1
    int mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      mine[j] = s_hist[kBins - 1 - (tid * kPer + j)];
      sum += mine[j];
    }
    int above = sum, unused = 0;
    block_before<THREADS>(above, unused, s_warp);
#pragma unroll
    for (int j = 0; j < kPer; ++j) s_hist[kBins - 1 - (tid * kPer + j)] = 0;
    if (above < want && want <= above + sum) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        if (above < want && want <= above + mine[j]) {
          s_digit = kBins - 1 - (tid * kPer + j);
          s_left = want - above;
          s_in = mine[j];
        }
        above += mine[j];
      }
    }
    if (tid == 0) s_listed = 0;
    __syncthreads();
    found |= (uint32_t)s_digit << shift;
    want = s_left;   // so many of the keys that begin like this one stay
    if (pass == 2) break;
    const int was = shift, next = pass == 0 ? 10 : 0;
    auto count = [&](uint32_t k) { atomicAdd(&s_hist[(k >> next) & (pass == 0 ? 2047u : 1023u)], 1); };
    if (listed) {
      for (int i = tid; i < listed; i += THREADS)
        if ((s_list[i] >> was) == (found >> was)) count(s_list[i]);
    } else {
      const bool list = s_in <= kListMost;
      for (int q = q0 + tid; q < q1; q += THREADS) {
        const uint4 four = keys(q);
        const uint32_t k[4] = {four.x, four.y, four.z, four.w};
        unsigned like = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) like |= (unsigned)((k[j] ^ found) >> was == 0u) << j;
        like &= members(q);
        for (; like; like &= like - 1) {
          const int j = __ffs(like) - 1;
          const uint32_t x = j & 2 ? (j & 1 ? k[3] : k[2]) : (j & 1 ? k[1] : k[0]);
          if (list) s_list[atomicAdd(&s_listed, 1)] = x;
          count(x);
        }
      }
      __syncthreads();
      if (list) listed = s_listed;
    }
    shift = next;
  }
  // ---- the positions, in order: thread t has `per` fours from the t * per-th on, as bits of a word ----
  const int per = min(7, ((q1 - q0 + THREADS - 1) / THREADS) | 1);   // (odd: no conflicts in shared memory)
  int at0 = first, eq0 = 0;   // places taken by higher ones before these fours; equal ones before them
  for (int s0 = q0; s0 < q1; s0 += THREADS * per) {
    const int b = min(q1, s0 + tid * per), cnt = min(q1 - b, per);
    unsigned higher = 0, same = 0;
    for (int i = 0; i < cnt; ++i) {
      const uint4 four = keys(b + i);
      const unsigned in = members(b + i);
      unsigned g = (unsigned)(four.x > found) | (unsigned)(four.y > found) << 1 | (unsigned)(four.z > found) << 2 |
                   (unsigned)(four.w > found) << 3;
      unsigned e = (unsigned)(four.x == found) | (unsigned)(four.y == found) << 1 | (unsigned)(four.z == found) << 2 |
                   (unsigned)(four.w == found) << 3;
      higher |= (g & in) << (4 * i);
      same |= (e & in) << (4 * i);
    }
    int gt = __popc(higher), eq = __popc(same);
    const int2 all = block_before<THREADS>(gt, eq, s_warp);
    const int room = want - eq0 - eq;                         // of the equal ones, the first stay
    while (__popc(same) > max(room, 0)) same &= ~(0x80000000u >> __clz(same));
    int at = at0 + gt + min(eq0 + eq, want);
    for (unsigned m = higher | same; m; m &= m - 1) kept[at++] = 4 * b + __ffs(m) - 1;
    at0 += all.x;
    eq0 += all.y;
    __syncthreads();   // (the sums' place is free)
  }
}

// ---------------------------------------------------------------- compaction
// Row i of a request's kept ones goes to position i, from a position that is never smaller: what is written in a round
// (rows of consecutive i) has been read in it or in one before, and no later round reads there.  So the rows pass through
// shared memory in rounds: a round's rows are written when all of the CTA's threads have theirs, while the next three
// rounds' are on their way.  K and V of a (request, KV head) are CTAs of their own, and where these do not fill the GPU, so
// are the halves or quarters of the channels, which need not wait for one another either.  The places of 2048 rows are found
// at once: found round by round, two dependent reads each, they held the rows up (16 requests of 5000-8192 tokens to 2048,
// 8 KV heads: 76 us, whether the rows lay scattered or side by side).
// Bound: HBM (a row that moves is read once and written once): 16 requests of 5000-8192 tokens to 2048, 8 KV heads, 52 us, 79 %.
constexpr int kMoveThreads = 256, kMoveStages = 4, kMoveSteps = 4;
constexpr int kMoveStage = kMoveSteps * kMoveThreads * 16;   // bytes of a round
constexpr int kMoveSeg = 2048;                               // rows whose places are known
constexpr int kMoveSmem = kMoveStages * kMoveStage + 2 * kMoveSeg * 8;
constexpr uint64_t kNowhere = ~0ull;
constexpr int kGiveBlocks = 16;                              // that put pages back

struct CompactArgs {
  char *k, *v;
  long long sp, st, sh;            // strides in bytes
  const int32_t *table, *kv_len, *kept, *kept_len;
  float* scores;                   // may be null
  int32_t* free_pages;             // may be null
  const int32_t* free_state;
  int32_t* free_out;
  int n_free, n_req, width, page_log2, n_pages, h_kv, max_keep;
  int n_give;                      // blocks that put pages back
};

// A request's tokens and those that it keeps; false: it stays as it is.
__device__ __forceinline__ bool load_kept(const CompactArgs& a, int r, int* n, int* len) {
  *n = clamp_len(a.kv_len[r], a.width, a.page_log2);
  *len = max(a.kept_len[r], 0);
  return *len < *n && *len <= a.max_keep;
}
// The table's columns of request r whose pages lie behind its kept tokens.
__device__ __forceinline__ int2 left_over(const CompactArgs& a, int r) {
  int n, len;
  if (!load_kept(a, r, &n, &len)) return make_int2(0, 0);
  const int size = 1 << a.page_log2;
  return make_int2((len + size - 1) >> a.page_log2, (n + size - 1) >> a.page_log2);
}

// Requests whose pages a block puts back: enough for some 16 blocks at most, each of which counts what comes behind its own.
__device__ __host__ __forceinline__ int give_share(int n_req) { return (n_req + kGiveBlocks - 1) / kGiveBlocks; }
// The pages behind the kept tokens, put back in front of the free ones, request by request; entries that are no page (where
// the free list had run out) are not.  Block i has requests i * share on and stores theirs from the last one to the first:
// the list's end is known beforehand, its beginning is not.  The columns of 256 requests at a time are laid end to end, a
// thread to an entry: 1024 requests of 1024 tokens to 512 move in 96 us with or without lists (a CTA to a request behind all
// others: 101), 25000 pages of one request go back in 20.
__device__ __forceinline__ void give_back(const CompactArgs& a, int block, char* smem) {
  constexpr int kWarps = kMoveThreads / 32, kDeep = 8;
  long long* first = reinterpret_cast<long long*>(smem);              // [256] entries of the requests before
  long long* s_warp = first + kMoveThreads;                           // [8]
  int* col = reinterpret_cast<int*>(s_warp + kWarps);                 // [256] their first columns
  int* s_count = col + kMoveThreads;                                  // [8][8]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int share = give_share(a.n_req), r0 = min(a.n_req, block * share), r1 = min(a.n_req, r0 + share);
  const int next = min(max(a.free_state[0], 0), a.n_free);
  auto is_page = [&](int page) { return page >= 0 && page < a.n_pages; };
  auto lay_out = [&](int t0, int t1) {   // of requests t0 .. t1 - 1, 256 at most; how many there are
    const int2 cols = t0 + tid < t1 ? left_over(a, t0 + tid) : make_int2(0, 0);
    const long long mine = cols.y - cols.x;
    long long x = mine, all = 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += u;
    }
    __syncthreads();   // (those before have been read)
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    x -= mine;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) x += s_warp[w];
      all += s_warp[w];
    }
    first[tid] = x;
    col[tid] = cols.x;
    __syncthreads();
    return all;
  };
  auto entry = [&](int t0, int t1, long long e) {
    int lo = 0, hi = t1 - t0;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (first[m] <= e) lo = m; else hi = m;
    }
    return a.table[(long long)(t0 + lo) * a.width + col[lo] + (e - first[lo])];
  };
  int behind = 0;   // pages of the requests behind, this thread's
  for (int t0 = r1; t0 < a.n_req; t0 += kMoveThreads) {
    const int t1 = min(a.n_req, t0 + kMoveThreads);
    const long long all = lay_out(t0, t1);
#pragma unroll 4
    for (long long e = tid; e < all; e += kMoveThreads) behind += is_page(entry(t0, t1, e));
  }
  behind = __reduce_add_sync(0xffffffffu, behind);
  __syncthreads();
  if (lane == 0) s_count[warp] = behind;
  __syncthreads();
  int end = next;   // places from here on are taken
#pragma unroll
  for (int w = 0; w < kWarps; ++w) end -= s_count[w];
  for (int t1 = r1; t1 > r0; t1 -= kMoveThreads) {
    const int t0 = max(r0, t1 - kMoveThreads);
    for (long long e1 = lay_out(t0, t1); e1 > 0; e1 -= kDeep * kMoveThreads) {   // eight entries a thread, the last ones first
      int page[kDeep];
      unsigned on[kDeep];
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const long long e = e1 - 1 - u * kMoveThreads - tid;
        page[u] = e >= 0 ? entry(t0, t1, e) : -1;
      }
      __syncthreads();   // (the counts before have been read)
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        on[u] = __ballot_sync(0xffffffffu, is_page(page[u]));
        if (lane == 0) s_count[u * kWarps + warp] = __popc(on[u]);
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        int at = end - 1 - __popc(on[u] & ((1u << lane) - 1u));
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const int n = s_count[u * kWarps + w];
          if (w < warp) at -= n;
          end -= n;
        }
        if (is_page(page[u]) && at >= 0) a.free_pages[at] = page[u];
      }
    }
  }
  if (block == 0 && tid == 0) {
    a.free_out[0] = max(0, end);
    a.free_out[1] = min(a.free_state[1], a.n_free);
    a.free_out[2] = max(0, -end);
  }
}

// Block: first those that give pages back (beside the others' work: as the last ones they took 67 us of their own with 1024
// requests), then ((request, KV head) * 2 + tensor) * PARTS + part of the channels.
template <int PARTS>
__global__ void __launch_bounds__(kMoveThreads, 2) k_page_compact(const CompactArgs a) {
  constexpr int kLanes = 16 / PARTS, kAtOnce = kMoveThreads / kLanes;   // threads to a row's part, rows to a step
  constexpr int kRows = kMoveSteps * kAtOnce;                           // of a round
  extern __shared__ __align__(16) char s_move[];                        // [stage][step][thread] 16 bytes
  uint64_t* s_from = reinterpret_cast<uint64_t*>(s_move + kMoveStages * kMoveStage);
  uint64_t* s_to = s_from + kMoveSeg;
  zc_let_next_start();
  zc_wait_for_last();
  const int block = (int)blockIdx.x - a.n_give;
  if (block < 0) {
    give_back(a, blockIdx.x, s_move);
    return;
  }
  const int tid = threadIdx.x, group = tid / kLanes;
  const int part = block % PARTS, c = block / PARTS;
  const int unit = c >> 1, r = unit / a.h_kv, head = unit - r * a.h_kv;
  const bool values = c & 1;
  int n, len;
  if (!load_kept(a, r, &n, &len)) return;
  const int32_t* table = a.table + (long long)r * a.width;
  const int32_t* kept = a.kept + (long long)unit * a.max_keep;
  char* pool = (values ? a.v : a.k) + head * a.sh + part * (256 / PARTS) + (tid % kLanes) * 16;
  const int mask = (1 << a.page_log2) - 1;
  const bool weighs = a.scores && !values && part == 0;
  const uint32_t score_bytes = 4u << a.page_log2;
  auto score_at = [&](int page, int row) {
    return reinterpret_cast<float*>(reinterpret_cast<char*>(a.scores) +
                                    (uint64_t)((uint32_t)page * (uint32_t)a.h_kv + head) * score_bytes + 4u * row);
  };
#pragma unroll 1
  for (int seg = 0; seg < len; seg += kMoveSeg) {
    const int cnt = min(kMoveSeg, len - seg);
    __syncthreads();   // the segment before has been written
    constexpr int kPer = kMoveSeg / kMoveThreads;
    int src[kPer], page[kPer], to[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = u * kMoveThreads + tid;
      src[u] = i < cnt ? kept[seg + i] : -1;
      to[u] = i < cnt ? table[(seg + i) >> a.page_log2] : -1;
      if (src[u] == seg + i || src[u] >= n || to[u] < 0 || to[u] >= a.n_pages) src[u] = -1;   // stays where it is
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      page[u] = src[u] >= 0 ? table[src[u] >> a.page_log2] : -1;
      if (page[u] >= a.n_pages) page[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = u * kMoveThreads + tid;
      if (i >= cnt) break;
      s_from[i] = page[u] >= 0 ? (uint32_t)page[u] * (uint64_t)a.sp + (uint32_t)(src[u] & mask) * (uint64_t)a.st : kNowhere;
      s_to[i] = (uint32_t)max(to[u], 0) * (uint64_t)a.sp + (uint32_t)((seg + i) & mask) * (uint64_t)a.st;
    }
    float score[kPer];
    if (weighs)
#pragma unroll
      for (int u = 0; u < kPer; ++u)
        if (page[u] >= 0) score[u] = *score_at(page[u], src[u] & mask);
    __syncthreads();
    if (weighs)
#pragma unroll
      for (int u = 0; u < kPer; ++u)
        if (page[u] >= 0) *score_at(to[u], (seg + u * kMoveThreads + tid) & mask) = score[u];
    auto ask = [&](int round) {
      char* at = s_move + (round % kMoveStages) * kMoveStage + tid * 16;
#pragma unroll
      for (int t = 0; t < kMoveSteps; ++t) {
        const int i = round * kRows + t * kAtOnce + group;
        const uint64_t from = i < cnt ? s_from[i] : kNowhere;
        if (from != kNowhere) zc_cp_async16(at + t * (kMoveThreads * 16), pool + from);
      }
    };
    const int rounds = (cnt + kRows - 1) / kRows;
#pragma unroll
    for (int i = 0; i < kMoveStages - 1; ++i) {
      if (i < rounds) ask(i);
      zc_cp_async_commit();
    }
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
      if (round + kMoveStages - 1 < rounds) ask(round + kMoveStages - 1);
      zc_cp_async_commit();
      zc_cp_async_wait<kMoveStages - 1>();
      __syncthreads();   // every thread has its pieces of this round
      const char* at = s_move + (round % kMoveStages) * kMoveStage + tid * 16;
#pragma unroll
      for (int t = 0; t < kMoveSteps; ++t) {
        const int i = round * kRows + t * kAtOnce + group;
        if (i < cnt && s_from[i] != kNowhere)
          *reinterpret_cast<uint4*>(pool + s_to[i]) = *reinterpret_cast<const uint4*>(at + t * (kMoveThreads * 16));
      }
    }
  }
}

template <int THREADS>
cudaError_t launch_select(const SelectArgs& a, int units, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = zc_allow_smem(k_page_select<THREADS>, kSelectRoom - kSelectFixed, &allowed);
  if (e != cudaSuccess) return e;
  return zc_launch_early(k_page_select<THREADS>, dim3(units), dim3(THREADS), (size_t)a.held * 16, st, a);
}
template <int PARTS>
cudaError_t launch_compact(const CompactArgs& a, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = zc_allow_smem(k_page_compact<PARTS>, kMoveSmem, &allowed);
  if (e != cudaSuccess) return e;
  const int grid = 2 * PARTS * a.n_req * a.h_kv + a.n_give;
  return zc_launch_early(k_page_compact<PARTS>, dim3((unsigned)grid), dim3(kMoveThreads), kMoveSmem, st, a);
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
struct Span { const void* at; long long bytes; };
bool overlap(const Span& a, const Span& b) {
  const char *x = (const char*)a.at, *y = (const char*)b.at;
  return x && y && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

}  // namespace

extern "C" {

int zc_page_select(zc_pages* p, const int32_t* table, int table_width, const int32_t* kv_len, int n_req,
                   const float* scores, const int32_t* keep, int recent, const int32_t* first, int32_t* kept,
                   int max_keep, int32_t* kept_len, zc_stream_t stream) {
  if (!p || n_req < 0 || recent < 0 || max_keep < 0) return ZC_EINVAL;
  if (n_req == 0) return ZC_OK;
  if (!table || !kv_len || !scores || !keep || (!kept && max_keep) || !kept_len || table_width < 1) return ZC_EINVAL;
  const long long cap = (long long)table_width << p->page_log2, units = (long long)n_req * p->cfg.n_kv_heads;
  if (cap > ZC_NO_WINDOW || units > 0x7fffffffLL) return ZC_EINVAL;
  if (!aligned4(table) || !aligned4(kv_len) || !aligned16(scores) || !aligned4(keep) || !aligned4(first) ||
      !aligned4(kept) || !aligned4(kept_len))
    return ZC_EALIGN;
  const Span in[5] = {{table, 4LL * n_req * table_width}, {kv_len, 4LL * n_req}, {keep, 4LL * n_req},
                      {first, 4LL * n_req}, {scores, (4LL * p->cfg.n_pages * p->cfg.n_kv_heads) << p->page_log2}};
  const Span out[2] = {{kept, 4LL * units * max_keep}, {kept_len, 4LL * n_req}};
  for (const Span& i : in)
    for (const Span& o : out)
      if (overlap(i, o)) return ZC_EINVAL;
  if (overlap(out[0], out[1])) return ZC_EINVAL;
  SelectArgs a;
  a.table = table;
  a.kv_len = kv_len;
  a.keep = keep;
  a.first = first;
  a.scores = scores;
  a.kept = kept;
  a.kept_len = kept_len;
  a.width = table_width;
  a.page_log2 = p->page_log2;
  a.n_pages = p->cfg.n_pages;
  a.h_kv = p->cfg.n_kv_heads;
  a.recent = recent;
  a.max_keep = max_keep;
  // as many keys in shared memory as leave room for the CTAs that an SM has to take, four at most (2048 threads)
  const long long per_sm = (units + p->n_sm - 1) / p->n_sm;
  const long long room = (kSelectRoom / (per_sm < 4 ? per_sm : 4) - kSelectFixed) / 16;
  const long long fours = cap / 4 + 1;   // (the candidates may begin inside a four)
  a.held = (int)(fours < room ? fours : room);
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = cap <= 2048 ? launch_select<256>(a, (int)units, st) : launch_select<512>(a, (int)units, st);
  p->launches += 1;
  return zc_cuda_status((int)e);
}

int zc_page_compact(zc_pages* p, const int32_t* table, int table_width, const int32_t* kv_len, int n_req,
                    const int32_t* kept, int max_keep, const int32_t* kept_len, float* scores, int32_t* free_pages,
                    int n_free, const int32_t* free_state, int32_t* free_out, zc_stream_t stream) {
  if (!p || n_req < 0 || max_keep < 0 || n_free < 0) return ZC_EINVAL;
  if (n_req == 0) return ZC_OK;
  if (!table || !kv_len || (!kept && max_keep) || !kept_len || table_width < 1) return ZC_EINVAL;
  const bool lists = free_pages || free_state || free_out;
  if (lists && (!free_pages || !free_state || !free_out)) return ZC_EINVAL;
  const long long units = (long long)n_req * p->cfg.n_kv_heads;
  if ((long long)table_width << p->page_log2 > ZC_NO_WINDOW || units * 9 > 0x7fffffffLL) return ZC_EINVAL;
  if (!aligned4(table) || !aligned4(kv_len) || !aligned4(kept) || !aligned4(kept_len) || !aligned4(scores) ||
      !aligned4(free_pages) || !aligned4(free_state) || !aligned4(free_out))
    return ZC_EALIGN;
  // every CTA reads the lengths, the table and the lists, some after others have written
  const Span in[5] = {{table, 4LL * n_req * table_width}, {kv_len, 4LL * n_req}, {kept, 4LL * units * max_keep},
                      {kept_len, 4LL * n_req}, {free_state, 12}};
  const Span out[3] = {{scores, (4LL * p->cfg.n_pages * p->cfg.n_kv_heads) << p->page_log2},
                       {free_pages, 4LL * n_free}, {free_out, 12}};
  for (int i = 0; i < 5; ++i)
    for (int o = 0; o < 3; ++o)
      if (overlap(in[i], out[o])) return ZC_EINVAL;
  if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return ZC_EINVAL;
  CompactArgs a;
  const int64_t* s = p->cfg.strides;
  a.k = p->k;
  a.v = p->v;
  a.sp = 2 * s[0];
  a.st = 2 * s[1];
  a.sh = 2 * s[2];
  a.table = table;
  a.kv_len = kv_len;
  a.kept = kept;
  a.kept_len = kept_len;
  a.scores = scores;
  a.free_pages = free_pages;
  a.free_state = free_state;
  a.free_out = free_out;
  a.n_free = n_free;
  a.n_req = n_req;
  const int share = give_share(n_req);
  a.n_give = free_pages ? (n_req + share - 1) / share : 0;
  a.width = table_width;
  a.page_log2 = p->page_log2;
  a.n_pages = p->cfg.n_pages;
  a.h_kv = p->cfg.n_kv_heads;
  a.max_keep = max_keep;
  // Whole rows where K and V of all units come to about two CTAs per SM, else as many parts as give that (measured at
  // 2048 of 8192 tokens, whole rows / halves / quarters: 128 units 58 / 62 / 70 us, 64 units 38 / 30 / 36; 8 units, 16384 of
  // 32768 tokens, 167 / 105 / 96).
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = 5 * units >= 4 * p->n_sm   ? launch_compact<1>(a, st)
                        : 5 * units >= 2 * p->n_sm ? launch_compact<2>(a, st)
                                                   : launch_compact<4>(a, st);
  p->launches += 1;
  return zc_cuda_status((int)e);
}

}  // extern "C"
