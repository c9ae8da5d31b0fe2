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
// memory (49152 of them; the rest is fetched again where it is needed).  The k-th largest is found digit by digit (11,
// 11 and 10 bits) in a histogram of 2048 places; then every warp counts its own stretch of positions, and writes the
// kept ones behind those of the warps before it, so that the list ascends.  Of the candidates equal to the k-th the
// first ones are kept.  Bound: latency (one read of the scores, three scans of the histogram).
constexpr int kBins = 2048;
constexpr int kSelMost = 49152;

// NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if (x != x) return 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

struct SelectArgs {
  const int32_t *table, *kv_len, *keep, *first;
  const float* scores;
  int32_t *kept, *kept_len;
  int width, page_log2, n_pages, h_kv, recent, max_keep, held;   // held: keys that shared memory has room for
};

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_page_select(const SelectArgs a) {
  constexpr int kWarps = THREADS / 32, kPer = kBins / THREADS;
  extern __shared__ uint32_t s_keys[];
  __shared__ int s_hist[kBins];
  __shared__ int s_warp[2][kWarps];
  __shared__ int s_digit, s_left;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r = blockIdx.x / a.h_kv, head = blockIdx.x - r * a.h_kv;
  zc_let_next_start();
  zc_wait_for_last();
  const int n = clamp_len(a.kv_len[r], a.width, a.page_log2);
  const int first = a.first ? min(max(a.first[r], 0), n) : 0;
  const int recent = min(a.recent, n - first);
  const int budget = max(min(max(a.keep[r], 0), a.max_keep), first + recent);
  const bool whole = budget >= n || budget > a.max_keep;   // nothing is evicted
  const int len = whole ? n : budget;
  int32_t* kept = a.kept + (long long)blockIdx.x * a.max_keep;
  if (head == 0 && tid == 0) a.kept_len[r] = len;
  for (int i = min(len, a.max_keep) + tid; i < a.max_keep; i += THREADS) kept[i] = -1;
  if (whole) {
    for (int i = tid; i < min(n, a.max_keep); i += THREADS) kept[i] = i;
    return;
  }
  const int c0 = first, nc = n - recent - first;   // candidates: nc positions from c0 on
  int want = budget - first - recent;              // of which so many stay, fewer than nc
  const int32_t* table = a.table + (long long)r * a.width;
  auto fetch = [&](int i) {
    const int t = c0 + i, page = table[t >> a.page_log2];
    if (page < 0 || page >= a.n_pages) return 0u;
    return score_key(a.scores[(((long long)page * a.h_kv + head) << a.page_log2) + (t & ((1 << a.page_log2) - 1))]);
  };
  auto key = [&](int i) { return i < a.held ? s_keys[i] : fetch(i); };
  // ---- the want-th largest key ----
  uint32_t found = 0;
  int shift = 21;
#pragma unroll 1
  for (int pass = 0; pass < 3 && want > 0; ++pass) {
    const int bits = pass < 2 ? 11 : 10;
    for (int i = tid; i < kBins; i += THREADS) s_hist[i] = 0;
    __syncthreads();
    auto count = [&](bool on, uint32_t k) {
      // many tokens of one weight (none yet, say) are one addition of the warp's
      const uint32_t bin = (k >> shift) & ((1u << bits) - 1);
      const unsigned some = __ballot_sync(0xffffffffu, on);
      if (some == 0xffffffffu) {
        int same;
        __match_all_sync(0xffffffffu, bin, &same);
        if (same) {
          if (lane == 0) atomicAdd(&s_hist[bin], 32);
          return;
        }
      }
      if (on) atomicAdd(&s_hist[bin], 1);
    };
    if (pass == 0) {
      constexpr int kUnroll = 8;
      for (int i0 = 0; i0 < nc; i0 += kUnroll * THREADS) {
        uint32_t k[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int i = i0 + u * THREADS + tid;
          k[u] = i < nc ? fetch(i) : 0u;
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int i = i0 + u * THREADS + tid;
          if (i0 + u * THREADS >= nc) break;
          if (i < nc && i < a.held) s_keys[i] = k[u];
          count(i < nc, k[u]);
        }
      }
    } else {
      for (int i0 = 0; i0 < nc; i0 += THREADS) {
        const int i = i0 + tid;
        const uint32_t k = i < nc ? key(i) : 0u;
        count(i < nc && (k >> (shift + bits)) == (found >> (shift + bits)), k);
      }
    }
    __syncthreads();
    // places from the top: thread t has the kPer places below those of thread t - 1
    int mine[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      mine[j] = s_hist[kBins - 1 - (tid * kPer + j)];
      sum += mine[j];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) s_warp[0][warp] = incl;
    __syncthreads();
    int above = incl - sum;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
      if (w < warp) above += s_warp[0][w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (above < want && want <= above + mine[j]) {
        s_digit = kBins - 1 - (tid * kPer + j);
        s_left = want - above;
      }
      above += mine[j];
    }
    __syncthreads();
    found |= (uint32_t)s_digit << shift;
    want = s_left;   // so many of the keys that begin like this one stay
    shift -= pass == 0 ? 11 : 10;
  }
  // ---- the positions, in order: warp w has candidates from w * stretch on ----
  const bool some = budget > first + recent;       // else no candidate stays
  const int stretch = (nc + THREADS - 1) / THREADS * 32;
  const int b = min(nc, warp * stretch), e = min(nc, b + stretch);
  int gt = 0, eq = 0;
  if (some) {
    for (int i0 = b; i0 < e; i0 += 32) {
      const uint32_t k = i0 + lane < e ? key(i0 + lane) : 0u;
      const bool in = i0 + lane < e;
      gt += __popc(__ballot_sync(0xffffffffu, in && k > found));
      eq += __popc(__ballot_sync(0xffffffffu, in && k == found));
    }
    if (lane == 0) {
      s_warp[0][warp] = gt;
      s_warp[1][warp] = eq;
    }
    __syncthreads();
    gt = eq = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
      if (w < warp) {
        gt += s_warp[0][w];
        eq += s_warp[1][w];
      }
    for (int i0 = b; i0 < e; i0 += 32) {
      const bool in = i0 + lane < e;
      const uint32_t k = in ? key(i0 + lane) : 0u;
      const unsigned g = __ballot_sync(0xffffffffu, in && k > found), q = __ballot_sync(0xffffffffu, in && k == found);
      const unsigned before = (1u << lane) - 1u;
      const int eq_here = eq + __popc(q & before), at = first + gt + __popc(g & before) + min(eq_here, want);
      if (in && (k > found || (k == found && eq_here < want))) kept[at] = c0 + i0 + lane;
      gt += __popc(g);
      eq += __popc(q);
    }
  }
  for (int i = tid; i < first; i += THREADS) kept[i] = i;
  for (int i = tid; i < recent; i += THREADS) kept[len - recent + i] = n - recent + i;
}

// ---------------------------------------------------------------- compaction
// Row i of a request's kept ones goes to position i, from a position that is never smaller: what is written in a round
// (rows of consecutive i) has been read in it or in one before, and no later round reads there.  So a round is: every
// thread of the cluster has its pieces of rows in registers; the cluster meets; all write.  K and V of a (request, KV
// head) are clusters of their own; a cluster is 1 to 8 CTAs, as many as fill the GPU: with few requests the rounds
// would otherwise follow one another in a few CTAs.  Bound: HBM (a row that moves is read once and written once).
constexpr int kMoveThreads = 256, kMoveUnroll = 8;
constexpr int kMoveRows = kMoveThreads / 16 * kMoveUnroll;   // rows of a CTA's round
constexpr int kMoveCluster = 8;

struct CompactArgs {
  char *k, *v;
  long long sp, st, sh;            // strides in bytes
  const int32_t *table, *kv_len, *kept, *kept_len;
  float* scores;                   // may be null
  int32_t* free_pages;             // may be null
  const int32_t* free_state;
  int32_t* free_out;
  int n_free, n_req, width, page_log2, n_pages, h_kv, max_keep, cluster;
};

// A request's tokens and those that it keeps; false: it stays as it is.
__device__ __forceinline__ bool load_kept(const CompactArgs& a, int r, int* n, int* len) {
  *n = clamp_len(a.kv_len[r], a.width, a.page_log2);
  *len = max(a.kept_len[r], 0);
  return *len < *n && *len <= a.max_keep;
}
__device__ __forceinline__ int pages_left_over(const CompactArgs& a, int r) {
  int n, len;
  if (!load_kept(a, r, &n, &len)) return 0;
  const int size = 1 << a.page_log2;
  return ((n + size - 1) >> a.page_log2) - ((len + size - 1) >> a.page_log2);
}

__global__ void __launch_bounds__(kMoveThreads) k_page_compact(const CompactArgs a) {
  __shared__ int s_sum[2];
  const int part = (threadIdx.x & 15) * 16, group = threadIdx.x >> 4;
  const int rank = blockIdx.x % a.cluster, c = blockIdx.x / a.cluster;
  const int unit = c >> 1, r = unit / a.h_kv, head = unit - r * a.h_kv;
  const bool values = c & 1;
  zc_let_next_start();
  zc_wait_for_last();
  const int32_t* table = a.table + (long long)r * a.width;
  // ---- the pages behind the kept tokens, put back in front of the free ones: one CTA per request ----
  if (a.free_pages && values && head == 0 && rank == 0) {
    if (threadIdx.x < 2) s_sum[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.n_req; i += kMoveThreads) {
      const int gone = pages_left_over(a, i);
      if (gone) {
        atomicAdd(&s_sum[1], gone);
        if (i < r) atomicAdd(&s_sum[0], gone);
      }
    }
    __syncthreads();
    const int total = s_sum[1], mine = pages_left_over(a, r);
    const int next = min(max(a.free_state[0], 0), a.n_free);
    const int at = next - total + s_sum[0];
    const int stay = mine ? (max(a.kept_len[r], 0) + (1 << a.page_log2) - 1) >> a.page_log2 : 0;
    for (int i = threadIdx.x; i < mine; i += kMoveThreads)
      if (at + i >= 0) a.free_pages[at + i] = table[stay + i];
    if (r == 0 && threadIdx.x == 0) {
      a.free_out[0] = max(0, next - total);
      a.free_out[1] = min(a.free_state[1], a.n_free);
      a.free_out[2] = max(0, total - next);
    }
  }
  // ---- the rows ----
  int n, len;
  if (!load_kept(a, r, &n, &len)) return;   // (the whole cluster's)
  const int32_t* kept = a.kept + (long long)unit * a.max_keep;
  char* pool = (values ? a.v : a.k) + head * a.sh + part;
  const int mask = (1 << a.page_log2) - 1;
  const bool weighs = a.scores && !values && part == 0;
  const int step = a.cluster * kMoveRows;
#pragma unroll 1
  for (int i0 = rank * kMoveRows; i0 - rank * kMoveRows < len; i0 += step) {
    int src[kMoveUnroll], from[kMoveUnroll];
    uint4 x[kMoveUnroll];
    float s[kMoveUnroll];
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u) {
      const int i = i0 + u * (kMoveThreads / 16) + group;
      src[u] = i < len ? kept[i] : -1;
      if (src[u] == i || src[u] >= n) src[u] = -1;   // stays where it is
    }
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u) {
      from[u] = src[u] >= 0 ? table[src[u] >> a.page_log2] : -1;
      if (from[u] >= a.n_pages) from[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (from[u] >= 0) {
        x[u] = *reinterpret_cast<const uint4*>(pool + from[u] * a.sp + (src[u] & mask) * a.st);
        if (weighs) s[u] = a.scores[(((long long)from[u] * a.h_kv + head) << a.page_log2) + (src[u] & mask)];
      }
    if (a.cluster > 1) {
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    } else {
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kMoveUnroll; ++u)
      if (from[u] >= 0) {
        const int i = i0 + u * (kMoveThreads / 16) + group, page = table[i >> a.page_log2];
        if (page >= 0 && page < a.n_pages) {
          *reinterpret_cast<uint4*>(pool + page * a.sp + (i & mask) * a.st) = x[u];
          if (weighs) a.scores[(((long long)page * a.h_kv + head) << a.page_log2) + (i & mask)] = s[u];
        }
      }
  }
}

template <int THREADS>
cudaError_t launch_select(const SelectArgs& a, int units, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  cudaError_t e = zc_allow_smem(k_page_select<THREADS>, kSelMost * 4, &allowed);
  if (e != cudaSuccess) return e;
  return zc_launch_early(k_page_select<THREADS>, dim3(units), dim3(THREADS), (size_t)a.held * 4, st, a);
}

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
  if (!aligned4(table) || !aligned4(kv_len) || !aligned4(scores) || !aligned4(keep) || !aligned4(first) ||
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
  a.held = (int)(cap < kSelMost ? cap : kSelMost);
  const cudaError_t e = cap <= 2048 ? launch_select<256>(a, (int)units, (cudaStream_t)stream)
                                    : launch_select<512>(a, (int)units, (cudaStream_t)stream);
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
  if ((long long)table_width << p->page_log2 > ZC_NO_WINDOW || units * 2 * kMoveCluster > 0x7fffffffLL) return ZC_EINVAL;
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
  a.width = table_width;
  a.page_log2 = p->page_log2;
  a.n_pages = p->cfg.n_pages;
  a.h_kv = p->cfg.n_kv_heads;
  a.max_keep = max_keep;
  a.cluster = 1;
  while (a.cluster < kMoveCluster && 2 * units * a.cluster < 2 * p->n_sm) a.cluster *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * units * a.cluster));
  cfg.blockDim = dim3(kMoveThreads);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_page_compact, (const CompactArgs)a);
  p->launches += 1;
  return zc_cuda_status((int)e);
}

}  // extern "C"
