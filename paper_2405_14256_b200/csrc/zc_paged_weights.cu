// The weight that attention gives every cached token of a call, added up over the request's rows and the query heads of
// a KV head:  A[j, h] = sum over rows i of 2^(s_ij - lse_i),  s the scaled logits and lse the rows' log-sum-exp, base 2.
// The step's own tokens begin with it, older ones add it to what they have.  Every sum is formed by one thread in a
// fixed order, in fp32, and a slot is written by one thread of each request that scores it (one, if the caller leaves shared
// pages out): no atomics, the same bits every time.
//
// Single tokens: the attention kernel has left its logits beside the slots, k_score_add reads them once the log-sum-exp
// is known (4 bytes per key and query row instead of the key's 256).  Chunks: the logits are computed again on the
// tensor cores, k_chunk_weights.
#include <cstring>
#include <utility>
#include "zc_paged_tc.cuh"

namespace {

// A row without a log-sum-exp that sees keys has a logit that is NaN or +inf, or none above -inf: its weights are NaN.
__device__ __forceinline__ float or_nan(float lse) { return lse == -INFINITY ? __int_as_float(0x7fffffff) : lse; }
// min(x, 0), NaN where x is.
__device__ __forceinline__ float at_most_0(float x) {
  float y;
  asm("min.NaN.f32 %0, %1, 0f00000000;\n" : "=f"(y) : "f"(x));
  return y;
}

// ---------------------------------------------------------------- single tokens
// A thread has four consecutive slots of a page and KV head, whose R logits each lie beside each other.  What the kernels
// before it do not write (lengths, tables, old scores) is read for the first of its slots before it waits for them: they
// start it only when all that came before them is complete.  Bound: HBM, or L2 where the logits are still there: 32
// requests of 2048-4096, 32 heads, 255 us with the attention's, which takes 232 alone; 4 of 200-512, 8 KV heads, 10.3 and 7.4.
constexpr int kAddThreads = 256;

struct AddArgs {
  ZcPagedArgs a;
  const float* logits;
  float* scores;
  const int32_t* first;       // may be null; of each request, tokens before it have no score
  const int32_t *group_start, *shared_len;   // instead of first, by the request's group
  int n_groups;
  int per_req;                // CTAs to a request
};

// R: logits of a key (a.max_rows * G), each number with an instance of its own: one loop of single loads for any R took 24.9 us
// instead of 15.2 with 12 of them (4 requests of 200-512, the attention's 13 included), 132 instead of 103 with 15 (32 of 2048-4096).
template <int R>
__global__ void __launch_bounds__(kAddThreads) k_score_add(const AddArgs w) {
  const ZcPagedArgs& a = w.a;
  const int r = blockIdx.x / w.per_req, part = blockIdx.x - r * w.per_req;
  zc_let_next_start();
  const Chunk c = load_chunk(a, r);
  if (c.n <= 0) return zc_wait_for_last();   // (the whole block; what comes behind waits for this kernel alone)
  const int rows = c.n * a.G;
  int first = w.first ? max(w.first[r], 0) : 0;
  if (w.n_groups > 0) {
    int g = -1;   // the last group that begins at or before the request
    for (int i = 0; i <= w.n_groups; i += kAddThreads) {
      const int at = i + threadIdx.x;
      g += __syncthreads_count(at <= w.n_groups && w.group_start[at] <= r);
    }
    first = g >= 0 && g < w.n_groups ? max(w.shared_len[g], 0) : 0;
  }
  // (a row beyond the caller's bound is none of the call's; its token is)
  const ZcSeen s = zc_seen(c.p0, c.p0 + c.n - 1, a.window, a.sinks, a.page_log2);
  const int per_page = a.h_kv << (a.page_log2 - 2);               // threads to a page
  const int fb = first >> a.page_log2;                            // pages without a score
  const int skip = min(s.nb, min(fb, s.nsb) + max(0, fb - s.wb0));
  const long long total = (long long)(s.nb - skip) * per_page;
  bool waited = false;
  for (long long idx = (long long)part * kAddThreads + threadIdx.x; idx < total;
       idx += (long long)w.per_req * kAddThreads) {
    const int nth = total < (1LL << 32) ? (int)((uint32_t)idx / (uint32_t)per_page) : (int)(idx / per_page);
    const int e = (int)(idx - (long long)nth * per_page) * 4;     // slot of the page's, all heads
    const int vb = nth + skip;
    const int blk = vb < s.nsb ? vb : s.wb0 + vb - s.nsb;
    const int head = e >> a.page_log2, key = (blk << a.page_log2) + (e & ((1 << a.page_log2) - 1));
    if (key >= s.hi || key + 3 < first) continue;
    const int page = a.table[(long long)r * a.table_width + blk];
    if (page < 0 || page >= a.n_pages) continue;
    const long long slot = (((long long)page * a.h_kv) << a.page_log2) + e;
    const float* lse = a.lse + (long long)c.row0 * a.h_q + head * a.G;
    float4* at = reinterpret_cast<float4*>(w.scores + slot);
    const float4 old = *at;
    if (!waited) zc_wait_for_last();
    waited = true;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int row, const float (&x)[4]) {
      const int tok = a.max_rows == 1 ? 0 : row / a.G, p = c.p0 + tok;
      const float less = or_nan(lse[(long long)tok * a.h_q + row - tok * a.G]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool seen = key + k <= p && (key + k > p - a.window || key + k < a.sinks);
        // (a weight is at most 1: beyond 2^24 the logits' rounding alone would make it more)
        if (seen) sum[k] += zc_exp2(at_most_0(x[k] - less));
      }
    };
    float x[4 * R];
    const float4* from = reinterpret_cast<const float4*>(w.logits + slot * R);
#pragma unroll
    for (int i = 0; i < R; ++i) *reinterpret_cast<float4*>(x + 4 * i) = from[i];
#pragma unroll
    for (int row = 0; row < R; ++row) {
      const float of[4] = {x[row], x[R + row], x[2 * R + row], x[3 * R + row]};
      if (row < rows) add(row, of);
    }
    const float was[4] = {old.x, old.y, old.z, old.w};
    float now[4];
    bool all = true;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool on = key + k >= first && ((key + k >= s.lo && key + k < s.hi) || key + k < s.sink_n);
      now[k] = key + k >= c.p0 ? sum[k] : was[k] + sum[k];
      all = all && on;
      if (!on) now[k] = was[k];
    }
    if (all) {
      *at = make_float4(now[0], now[1], now[2], now[3]);
    } else {
      // slots that are not the request's, or that no row sees, may be another's by now
      float* one = reinterpret_cast<float*>(at);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (key + k >= first && ((key + k >= s.lo && key + k < s.hi) || key + k < s.sink_n)) one[k] = now[k];
    }
  }
  if (!waited) zc_wait_for_last();
}

// ---------------------------------------------------------------- chunks
// An item is 256 keys of one request and KV head.  Their two tiles of 128 stay in shared memory while the request's
// query rows that see any of them pass by in tiles of 128 rows (token * G + head), each multiplied with both:
// S = K Q^T, tcgen05, the keys as the rows of the product, so that a thread of group g owns a key of tile g and its sum
// needs no exchange.  Per tile of rows 2 x 128 x 128 exponentials: 2048 cycles of the exp2 unit, against 512 of the
// tensor cores and 32 KB of Q from L2 (with one tile of keys to an item it would be 32 KB per 1024 cycles).
//   warp 0      walks the items (a counter deals them out, long ones first), copies K (a lane per page) and Q
//   warp 1      issues the products, into two places of tensor memory per group
//   warp 2      brings the rows' log-sum-exp and positions to shared memory
//   warps 4-7, 8-11  groups 0 and 1, a key per thread: columns 0-63 of every tile
//   warps 12-15, 16-19  columns 64-127, whose sum the key's first thread gets at the item's end
// (With all 128 columns a thread, and two warps to a scheduler, the exp2 unit was 65 % busy.)
// Bound: the exp2 unit (68 % busy), the FMA pipe (53 %) and the issue slots (62 %) together: 289 us for 2048 rows behind 16000
// tokens, 32 over 8 heads, the tensor cores alone 172.
// Every wait is bounded; warps 0 to 2 leave where one runs out and wait for what they have in flight, the groups go on
// with void values until no more items come.  The blocks' warps meet at the kernel's end only.
constexpr int kThreads = 640;
constexpr int kKeys = 2 * kM;                          // keys of an item
constexpr int kKeysLog2 = 8;
constexpr int kKBufs = 2, kQBufs = 2, kLBufs = 4, kRing = 2;
constexpr int kTiles = (2 * kKBufs + kQBufs) * kTile;  // 192 KB
constexpr int kRowsBytes = kLBufs * (kM * 8 + 4);      // minus the log-sum-exp, position; mild
// The logits are the attention kernel's bit for bit, whatever their terms' sizes (the same products in the same order, with
// keys and rows in each other's place), so that a weight passes 1 by the log-sum-exp's rounding alone, 2^-24 of it: up to
// here by 2^0.07 at most.  Beyond, weights are held to 1.
constexpr float kMild = 1048576.f;
constexpr int kItemInts = 16;
constexpr int kPartBytes = 2 * kKeys * 4;              // sums of the second halves of the columns, of two items
constexpr int kSmem = kTiles + 1024 + 512 + kPartBytes + kRowsBytes + kRing * kItemInts * 4;
constexpr uint32_t kCols = 512;

struct WeightArgs {
  ZcPagedArgs a;
  const float* lse;
  float* scores;
  const int32_t* first;
  unsigned* next;             // [2] items dealt out beyond the first of each CTA, CTAs that are done; zero between calls
  int tpt;
};

struct WItem {
  int r, kv, key0;            // r < 0: no more items
  int row0, n, p0;
  int qa, qe;                 // tiles of rows
  int lo, hi, sink_n;         // keys that any row sees
  int first, two;             // two: the second tile has keys that a row sees
};
static_assert(sizeof(WItem) <= kItemInts * 4, "an item fits its place in the ring");
// Whether any row of tile t (tpt tokens) sees a key of the item's tile g; the tiles that no row of it does cost nothing.
__device__ __forceinline__ bool tile_seen(const WItem& it, const ZcPagedArgs& a, int tpt, int t, int g) {
  const int key = it.key0 + g * kM, p_first = it.p0 + t * tpt, p_last = it.p0 + min(it.n, (t + 1) * tpt) - 1;
  return key < it.hi && key <= p_last && (key + kM - 1 > p_first - a.window || key < a.sinks);
}

// 2^x of two numbers on the FMA pipe, x <= 2^20: x is rounded to a whole number n by adding 1.5 * 2^23, whose lower bits
// then hold n, and the rest, of -1/2 .. 1/2, goes through a polynomial of degree 5 (least largest relative error, fitted by
// reweighted least squares: 1.6e-7 with these fp32 coefficients); n is added to the exponent.  Below 2^-126: 2^-126.
__device__ __forceinline__ float2 exp2_fma(float2 x) {
  const float2 big = make_float2(12582912.f, 12582912.f), back = make_float2(-12582912.f, -12582912.f);
  x = make_float2(fmaxf(x.x, -126.f), fmaxf(x.y, -126.f));
  const float2 t = add2(x, big), n = add2(t, back);
  const float2 f = fma2(n, make_float2(-1.f, -1.f), x);
  float2 p = fma2(make_float2(0.0013276470f, 0.0013276470f), f, make_float2(0.0096755410f, 0.0096755410f));
  p = fma2(p, f, make_float2(0.055507131f, 0.055507131f));
  p = fma2(p, f, make_float2(0.24022120f, 0.24022120f));
  p = fma2(p, f, make_float2(0.69314694f, 0.69314694f));
  p = fma2(p, f, make_float2(1.00000012f, 1.00000012f));
  return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)),
                     __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}
// add += the weights 2^(v * scale + less) of 32 columns; kFmaPairs of eight pairs of them on the FMA pipe, since the exp2 unit
// alone would take eight cycles of a warp's for each, and the instructions beside it two (the call with 0, 1, 2, 3 pairs: 805,
// 792, 783, 791 us).
constexpr int kFmaPairs = 2;
__device__ __forceinline__ void sum_weights(const float* v, const float4* less, float scale, float2 (&add)[2]) {
  const float2 sc = make_float2(scale, scale);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const float4 l = less[c];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float2 x = fma2(make_float2(v[4 * c + 2 * h], v[4 * c + 2 * h + 1]), sc,
                            h ? make_float2(l.z, l.w) : make_float2(l.x, l.y));
      const int pair = (2 * c + h) & 7;
      const float2 e = (pair * kFmaPairs) % 8 < kFmaPairs ? exp2_fma(x) : make_float2(zc_exp2(x.x), zc_exp2(x.y));
      add[h] = add2(add[h], e);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
    k_chunk_weights(const WeightArgs w, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  const ZcPagedArgs& a = w.a;
  const uint32_t raw_u = zc_smem_u32(smem_raw);
  const uint32_t base_u = (raw_u + 1023u) & ~1023u;
  char* base = smem_raw + (base_u - raw_u);
  const uint32_t k_addr = base_u, q_addr = base_u + 2 * kKBufs * kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + kTiles);
  uint64_t* k_full = bars;                   // [kKBufs] both key tiles of an item
  uint64_t* k_free = k_full + kKBufs;        // [kKBufs]
  uint64_t* q_full = k_free + kKBufs;        // [kQBufs]
  uint64_t* q_free = q_full + kQBufs;        // [kQBufs]
  uint64_t* l_full = q_free + kQBufs;        // [kLBufs] a tile's log-sum-exps
  uint64_t* l_free = l_full + kLBufs;        // [kLBufs] all sixteen warps are through with them
  uint64_t* s_done = l_free + kLBufs;        // [2][2] S_g in place
  uint64_t* s_free = s_done + 4;             // [2][2] the group has read it
  uint64_t* i_full = s_free + 4;             // [kRing]
  uint64_t* i_free = i_full + kRing;         // [kRing]
  uint64_t* x_full = i_free + kRing;         // [2][2] group g's second halves have left their sums, of every other item
  uint64_t* x_free = x_full + 4;             // [2][2] its first halves have read them
  uint64_t* drained = x_free + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  float* s_part = reinterpret_cast<float*>(base + kTiles + 512);         // [2][kKeys]
  float* s_lse = s_part + 2 * kKeys;                                     // [kLBufs][kM]
  int* s_pos = reinterpret_cast<int*>(s_lse + kLBufs * kM);              // [kLBufs][kM]
  int* s_mild = s_pos + kLBufs * kM;                                     // [kLBufs] no row's is beyond kMild
  int* ring = s_mild + kLBufs;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  zc_let_next_start();
  if (tid == 0) {
    for (int i = 0; i < kKBufs; ++i) {
      bar_init(&k_full[i], 1);
      bar_init(&k_free[i], 1);
    }
    for (int i = 0; i < kQBufs; ++i) {
      bar_init(&q_full[i], 1);
      bar_init(&q_free[i], 1);
    }
    for (int i = 0; i < kLBufs; ++i) {
      bar_init(&l_full[i], 1);
      bar_init(&l_free[i], 16);
    }
    for (int i = 0; i < 4; ++i) {
      bar_init(&s_done[i], 1);
      bar_init(&s_free[i], 8);
      bar_init(&x_full[i], 4);
      bar_init(&x_free[i], 4);
    }
    for (int i = 0; i < kRing; ++i) {
      bar_init(&i_full[i], 1);
      bar_init(&i_free[i], 18);   // the products, the log-sum-exps, sixteen worker warps
    }
    bar_init(drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(zc_smem_u32(tmem_slot)),
                 "r"(kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  // rows of a Q tile that no copy fills (G that does not divide 128) are zeros: their columns then weigh nothing
  for (int i = tid; i < (kM - w.tpt * a.G) * 2 * kQBufs * 8; i += kThreads) {
    const int chunk = i & 7, half = (i >> 3) & 1, row = w.tpt * a.G + (i >> 4) / kQBufs, buf = (i >> 4) % kQBufs;
    *reinterpret_cast<uint4*>(base + (2 * kKBufs + buf) * kTile + half * kKBlock + row * 128 + chunk * 16) = make_uint4(0, 0, 0, 0);
  }
  async_proxy_fence();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  zc_wait_for_last();

  uint32_t n_item = 0;   // items taken from the ring
  auto next_item = [&](WItem& it) {
    const uint32_t at = n_item % kRing;
    if (!warp_wait(&i_full[at], (n_item / kRing) & 1u)) return false;
    const int* src = ring + at * kItemInts;
    int* dst = reinterpret_cast<int*>(&it);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(WItem) / 4); ++i) dst[i] = src[i];
    __syncwarp();
    if (lane == 0) bar_arrive(&i_free[at]);
    ++n_item;
    return it.r >= 0;
  };

  if (warp == 0) {
    // ---- items; K and Q ----
    // requests 32 at a time, a lane each; items run request by request, the keys from the first on (which more rows
    // see), the heads innermost
    int r0 = -32, blocks = 0, incl = 0;
    long long before = 0, window_items = 0;   // items before these requests, and of them
    Chunk c;
    c.row0 = c.n = c.p0 = 0;
    ZcSeen s;
    int skip = 0, first = 0;
    auto find_item = [&](long long idx, WItem& it) {
      it.r = -1;
      while (idx >= before + window_items) {
        before += window_items;
        r0 += 32;
        if (r0 >= a.n_req) return;
        const int r = r0 + lane;
        c.n = 0;
        blocks = 0;
        if (r < a.n_req) {
          c = load_chunk(a, r);
          if (c.n > 0) {
            first = w.first ? max(w.first[r], 0) : 0;
            s = zc_seen(c.p0, c.p0 + c.n - 1, a.window, a.sinks, kKeysLog2);
            const int fb = first >> kKeysLog2;   // blocks of keys that have no score
            skip = min(s.nb, min(fb, s.nsb) + max(0, fb - s.wb0));
            blocks = s.nb - skip;
          }
        }
        incl = blocks;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += u;
        }
        window_items = (long long)__shfl_sync(0xffffffffu, incl, 31) * a.h_kv;
      }
      const long long in = idx - before;
      const int blk = (int)(in / a.h_kv), kv = (int)(in - (long long)blk * a.h_kv);
      const int src = __ffs(__ballot_sync(0xffffffffu, blk < incl)) - 1;
      auto of = [&](int v) { return __shfl_sync(0xffffffffu, v, src); };
      const int vb = blk - of(incl - blocks) + of(skip), nsb = of(s.nsb), wb0 = of(s.wb0);
      it.r = r0 + src;
      it.kv = kv;
      it.key0 = (vb < nsb ? vb : wb0 + vb - nsb) << kKeysLog2;
      it.row0 = of(c.row0);
      it.n = of(c.n);
      it.p0 = of(c.p0);
      it.lo = of(s.lo);
      it.hi = of(s.hi);
      it.sink_n = of(s.sink_n);
      it.first = of(first);
      it.two = it.key0 + kM < it.hi;
      // rows at positions p >= key0 see a key of the item, up to p = its last key + window - 1 (or all, for the sinks)
      const int ta = max(0, it.key0 - it.p0);
      long long te = it.n;
      if (a.window < ZC_NO_WINDOW && it.key0 >= a.sinks) te = min(te, (long long)it.key0 + kKeys - 1 + a.window - it.p0);
      it.qa = ta / w.tpt;
      it.qe = te > ta ? (int)((te + w.tpt - 1) / w.tpt) : it.qa;
    };
    uint32_t n = 0, n_k = 0, n_q = 0;
    bool ok = true;
    WItem it;
    auto announce = [&]() {
      const uint32_t place = n % kRing;
      if (n >= kRing && !warp_wait(&i_free[place], (n / kRing - 1) & 1u)) return false;
      if (lane == 0) {
        int* dst = ring + place * kItemInts;
        const int* src = reinterpret_cast<const int*>(&it);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(WItem) / 4); ++i) dst[i] = src[i];
        bar_arrive(&i_full[place]);
      }
      __syncwarp();
      ++n;
      return true;
    };
    const int rows = min(kM, 1 << a.page_log2);      // of a box
    long long idx = blockIdx.x;
    for (;;) {
      find_item(idx, it);
      ok = announce();
      if (!ok || it.r < 0) break;
      unsigned taken = 0;
      if (lane == 0) taken = atomicAdd(&w.next[0], 1u);
      // keys: lane i brings the i-th page (or half of one) of the item
      const uint32_t kb = n_k % kKBufs;
      ok = n_k < kKBufs || warp_wait(&k_free[kb], (n_k / kKBufs - 1) & 1u);
      if (!ok) break;
      const int boxes = kKeys / rows, pk0 = it.key0 + lane * rows;
      const bool on = lane < boxes && pk0 < it.hi;
      const uint32_t some = (uint32_t)__popc(__ballot_sync(0xffffffffu, on));
      int page = a.n_pages;                            // beyond the pool: arrives as zeros
      if (on) {
        const int id = a.table[(long long)it.r * a.table_width + (pk0 >> a.page_log2)];
        if (id >= 0 && id < a.n_pages) page = id;
      }
      if (lane == 0) expect_bytes(&k_full[kb], some * (uint32_t)rows * (ZC_D * 2));
      __syncwarp();
      if (on) {
        const uint32_t dst = k_addr + (kb * 2 + lane * rows / kM) * kTile + (lane * rows % kM) * 128;
        const int row = pk0 & ((1 << a.page_log2) - 1);
        page_copy(&kmap, dst, &k_full[kb], row, 0, it.kv, page);
        page_copy(&kmap, dst + kKBlock, &k_full[kb], row, 1, it.kv, page);
      }
      __syncwarp();
      ++n_k;
      for (int t = it.qa; ok && t < it.qe; ++t, ++n_q) {
        const uint32_t qb = n_q % kQBufs;
        ok = n_q < kQBufs || warp_wait(&q_free[qb], (n_q / kQBufs - 1) & 1u);
        if (!ok) break;
        if (lane == 0) {
          expect_bytes(&q_full[qb], (uint32_t)(w.tpt * a.G * ZC_D * 2));
          for (int half = 0; half < 2; ++half)
            q_copy(&qmap, q_addr + qb * kTile + half * kKBlock, &q_full[qb], half, it.kv * a.G, it.row0 + t * w.tpt, 0);
        }
        __syncwarp();
      }
      if (!ok) break;
      idx = (long long)gridDim.x + __shfl_sync(0xffffffffu, taken, 0);
    }
    for (uint32_t i = 0; i < kKBufs; ++i)
      if (n_k > i) drain(&k_full[i], ((n_k - 1 - i) / kKBufs) & 1u);
    for (uint32_t i = 0; i < kQBufs; ++i)
      if (n_q > i) drain(&q_full[i], ((n_q - 1 - i) / kQBufs) & 1u);
    if (lane == 0) {
      // the last CTA to come here leaves the counters as the next call wants them
      __threadfence();
      if (atomicAdd(&w.next[1], 1u) == gridDim.x - 1) {
        w.next[0] = 0;
        w.next[1] = 0;
      }
    }
  } else if (warp == 1) {
    // ---- products ----
    const uint32_t tm = (uint32_t)uniform((int)tmem);
    const uint32_t idesc = instr_desc<T>();
    uint32_t n_k = 0, n_q = 0, n_s[2] = {0, 0};
    bool ok = true;
    WItem it;
    while (ok && next_item(it)) {
      const uint32_t kb = n_k % kKBufs;
      ok = warp_wait(&k_full[kb], (n_k / kKBufs) & 1u);
      const int cnt = uniform(it.qe - it.qa);
      for (int t = 0; ok && t < cnt; ++t, ++n_q) {
        const uint32_t qb = n_q % kQBufs;
        ok = warp_wait(&q_full[qb], (n_q / kQBufs) & 1u);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (!uniform(tile_seen(it, a, w.tpt, it.qa + t, g))) continue;
          const uint32_t place = n_s[g] & 1u;
          ok = ok && (n_s[g] < 2 || warp_wait(&s_free[2 * g + place], (n_s[g] / 2 - 1) & 1u));
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            mma_tile(tm + (2 * g + place) * kM, k_addr + (kb * 2 + g) * kTile, q_addr + qb * kTile, idesc);
            mma_commit(&s_done[2 * g + place]);
          }
          __syncwarp();
          ++n_s[g];
        }
        if (ok && elect_one()) mma_commit(&q_free[qb]);
        __syncwarp();
      }
      if (ok && elect_one()) mma_commit(&k_free[kb]);
      __syncwarp();
      ++n_k;
    }
    if (n_s[0] > 0) {
      if (elect_one()) mma_commit(drained);
      __syncwarp();
      drain(drained, 0);
    }
  } else if (warp == 2) {
    // ---- the rows' log-sum-exp and positions, four columns a lane ----
    uint32_t n_l = 0;
    bool ok = true;
    WItem it;
    while (ok && next_item(it)) {
      for (int t = it.qa; ok && t < it.qe; ++t, ++n_l) {
        float less[4];
        int pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int col = 4 * lane + i, in = col / a.G, tok = t * w.tpt + in;
          const bool on = in < w.tpt && tok < it.n;
          less[i] = on ? -or_nan(w.lse[(long long)(it.row0 + tok) * a.h_q + it.kv * a.G + col - in * a.G]) : -INFINITY;
          pos[i] = on ? it.p0 + tok : -1;
        }
        bool mild = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) mild = mild && (fabsf(less[i]) < kMild || pos[i] < 0);
        mild = __all_sync(0xffffffffu, mild);
        const uint32_t at = n_l % kLBufs;
        ok = n_l < kLBufs || warp_wait(&l_free[at], (n_l / kLBufs - 1) & 1u);
        if (!ok) break;
        *reinterpret_cast<float4*>(s_lse + at * kM + 4 * lane) = make_float4(less[0], less[1], less[2], less[3]);
        *reinterpret_cast<int4*>(s_pos + at * kM + 4 * lane) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        if (lane == 0) s_mild[at] = mild;
        __syncwarp();
        if (lane == 0) bar_arrive(&l_full[at]);
      }
    }
  } else if (warp >= 4) {
    const int g = (warp >> 2) - 1 & 1, half = warp >= 12, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t tmem_g = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)g * 2 * kM + 64u * half;
    const float scale = kLog2e * rsqrtf((float)ZC_D);
    uint32_t n_l = 0, n_s = 0, n_x = 0;
    WItem it;
    while (next_item(it)) {
      const int first_key = it.key0 + g * kM, key = first_key + row;
      const bool work = g == 0 || it.two;
      const int window = key < a.sinks ? 0x7fffffff : a.window;   // a sink is seen from everywhere behind it
      // this thread's slot, and what it has; asked for now, used at the item's end
      const bool mine = half == 0 && key >= it.first && ((key >= it.lo && key < it.hi) || key < it.sink_n);
      float* at = nullptr;
      if (mine) {
        const int page = a.table[(long long)it.r * a.table_width + (key >> a.page_log2)];
        if (page >= 0 && page < a.n_pages)
          at = w.scores + (((long long)page * a.h_kv + it.kv) << a.page_log2) + (key & ((1 << a.page_log2) - 1));
      }
      const float old = at && key < it.p0 ? *at : 0.f;
      float sum = 0.f;
      for (int t = it.qa; t < it.qe; ++t, ++n_l) {
        const uint32_t lb = n_l % kLBufs;
        bar_wait(&l_full[lb], (n_l / kLBufs) & 1u);
        if (tile_seen(it, a, w.tpt, t, g)) {
          const uint32_t place = n_s & 1u, tmem_s = tmem_g + place * kM;
          bar_wait(&s_done[2 * g + place], (n_s >> 1) & 1u);
          ++n_s;
          tc_fence_after();
          // pairs that are not to be counted: rows behind the request's, rows before the key, keys behind the window
          const int tok0 = t * w.tpt, p_first = it.p0 + tok0, p_last = it.p0 + min(it.n, tok0 + w.tpt) - 1;
          const bool edge = tok0 + w.tpt > it.n || first_key + kM - 1 > p_first ||
                            (first_key <= p_last - a.window && first_key + kM > a.sinks) || !s_mild[lb];
          float2 add[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float4* less = reinterpret_cast<const float4*>(s_lse + lb * kM + 64 * half);
          const int4* where = reinterpret_cast<const int4*>(s_pos + lb * kM + 64 * half);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[32];
            tmem_ld32_nowait(v, tmem_s + 32 * h);
            tmem_wait32(v);
            if (h == 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) bar_arrive(&s_free[2 * g + place]);   // this warp has read its S
            }
            if (!edge) {
              sum_weights(v, less + 8 * h, scale, add);
            } else {
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float4 l = less[8 * h + c];
                const int4 p = where[8 * h + c];
                auto one = [&](float x, float m, int at_pos) {
                  const bool seen = at_pos >= key && at_pos - key < window;   // (-1: no row)
                  return seen ? zc_exp2(at_most_0(fmaf(x, scale, m))) : 0.f;
                };
                add[0] = add2(add[0], make_float2(one(v[4 * c], l.x, p.x), one(v[4 * c + 1], l.y, p.y)));
                add[1] = add2(add[1], make_float2(one(v[4 * c + 2], l.z, p.z), one(v[4 * c + 3], l.w, p.w)));
              }
            }
          }
          const float2 both = add2(add[0], add[1]);
          sum += both.x + both.y;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(&l_free[lb]);
      }
      if (!work) continue;
      const uint32_t x = 2 * g + (n_x & 1u);
      float* part = s_part + (n_x & 1u) * kKeys + g * kM + row;
      if (half) {
        if (n_x >= 2) bar_wait(&x_free[x], (n_x / 2 - 1) & 1u);
        *part = sum;
        __syncwarp();
        if (lane == 0) bar_arrive(&x_full[x]);
      } else {
        bar_wait(&x_full[x], (n_x / 2) & 1u);
        sum += *part;
        __syncwarp();
        if (lane == 0) bar_arrive(&x_free[x]);
        if (at) *at = old + sum;
      }
      ++n_x;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kCols) : "memory");
}

template <int... R>   // 0 ...
cudaError_t launch_add(std::integer_sequence<int, R...>, int per, const AddArgs& w, dim3 grid, cudaStream_t st) {
  cudaError_t e = cudaErrorInvalidValue;
  ((R + 1 == per ? (void)(e = zc_launch_early(k_score_add<R + 1>, grid, dim3(kAddThreads), 0, st, w)) : (void)0), ...);
  return e;
}

template <typename T>
cudaError_t launch_weights(zc_pages* p, const WeightArgs& w, const CUtensorMap& qmap, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = zc_allow_smem(k_chunk_weights<T>, kSmem, &allowed);
  if (e != cudaSuccess) return e;
  return zc_launch_early(k_chunk_weights<T>, dim3(p->n_sm), dim3(kThreads), kSmem, st, w, qmap, p->k128);
}

}  // namespace

int zc_launch_score_add(zc_pages* p, const ZcPagedArgs& a, const float* logits, float* scores, const int32_t* first,
                        const int32_t* group_start, const int32_t* shared_len, int n_groups, cudaStream_t st) {
  AddArgs w;
  memset(&w, 0, sizeof(w));
  w.a = a;
  w.logits = logits;
  w.scores = scores;
  w.first = first;
  w.group_start = group_start;
  w.shared_len = shared_len;
  w.n_groups = n_groups;
  // as many CTAs as the table's width asks for at most, eight per SM over all requests
  const long long most = ((((long long)a.table_width * a.h_kv) << (a.page_log2 - 2)) + kAddThreads - 1) / kAddThreads;
  long long gx = 8LL * p->n_sm / a.n_req;
  gx = gx < 1 ? 1 : gx > most ? most : gx;
  w.per_req = (int)gx;
  if (gx * a.n_req > 0x7fffffffLL) return (int)cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)(gx * a.n_req));
  const cudaError_t e = launch_add(std::make_integer_sequence<int, ZC_PAGED_ROWS>(), a.max_rows * a.G, w, grid, st);
  if (e == cudaSuccess) p->launches += 1;
  return (int)e;
}

int zc_launch_chunk_weights(zc_pages* p, const ZcPagedArgs& a, float* scores, const int32_t* first, char* ws, cudaStream_t st) {
  if (!zc_page_maps(p)) return (int)cudaErrorNotSupported;
  WeightArgs w;
  memset(&w, 0, sizeof(w));
  w.a = a;
  w.lse = a.lse;
  w.scores = scores;
  w.first = first;
  w.next = (unsigned*)ws + ZC_PAGED_MAX_CTAS;
  w.tpt = tokens_per_tile(a.G);
  CUtensorMap qmap;
  memset(&qmap, 0, sizeof(qmap));
  if (!make_q_map(&qmap, a.q, p->cfg.dtype, a.h_q, a.G, a.n_rows, 1, a.qs_head, a.qs_row, 0))
    return (int)cudaErrorNotSupported;
  const cudaError_t e = p->cfg.dtype == ZC_F16 ? launch_weights<__half>(p, w, qmap, st)
                                               : launch_weights<__nv_bfloat16>(p, w, qmap, st);
  if (e == cudaSuccess) p->launches += 1;
  return (int)e;
}

int zc_paged_weights_error_code(int* out) { return (int)cudaMemcpyFromSymbol(out, g_zc_tc_error, sizeof(int)); }
