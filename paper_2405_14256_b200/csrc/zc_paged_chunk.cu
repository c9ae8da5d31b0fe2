// Attention of chunks of new tokens over pages, and of whole prompts in dense tensors under a sliding
// window (Eq. 2 with its causal mask; bound: tensor cores, and one exp2 per visible pair).
//
// The query heads of a KV head are packed beside each other: row = token * G + head, 128 / G tokens to
// a tile of 128 rows, so that short chunks fill the tile, a key tile is read once for the whole group and
// little work falls on tiles that the causal mask or the window cuts.  A work item is one request's and
// KV head's rows of two such tiles (groups 0 and 1 take one each), or of one (the groups then take the
// even and the odd key tiles, and their results meet at the end), and the key tiles (64 keys) that any
// of its rows sees: those of the first `sinks` tokens, then those of the window.  The CTAs are
// persistent, one per SM; each works through items until there are none:
//   warp 2      walks the CTA's items, one ahead of the others, and copies V
//   warp 1      copies K, as warp 2 V, page by page: a box per page of 64 tokens or more, a lane per page and a
//               box per half of the channels below that
//   warps 0, 3  copy Q (a box per half of a tile's channels) and issue the matrix products of group 0 and 1,
//               tcgen05.mma with accumulators in tensor memory:
//               S_g = Q_g K^T (both K-major in shared memory), 128 x 64, and O_g += P_g V (P_g in tensor
//               memory over the first half of its S, V with its channels contiguous), 128 x 128
//   warps 4-7, 8-11  groups 0 and 1, one row per thread: running maximum (renewed, and O rescaled, when the
//               weights' sum shows it to be far behind) and sum in fp32, P rounded to the input type, output and
//               log-sum-exp
// Each group has two places for S, and S of a key tile is computed two tiles ahead: a group turns one S
// after the other into P without waiting for a product, and the tensor cores' work hides behind that of
// the groups (and the other way round).  With 128 keys to a tile and one place for S, the chain product -
// weights - product left either side idle half of the time (5000 cycles per 256 rows x 128 keys; now 3300).
// The next item's Q and first key tiles arrive while this one's output is written.
//   Every wait is bounded, also that of the two groups for each other.  Warps 0 to 3 leave where one runs out: they
// issue nothing more, wait (with the bound) for their own copies and products in flight, and meet the others at the
// kernel's end; a worker warp goes on with void values until no more items come.
//   What it takes (1.7 GHz): 1650 cycles per wide tile, of which the tensor cores alone need 1140 and the exp2 unit
// 1020; about 5500 more per item (its first and last tiles' masks, the last product, 3000 for the output).  A chunk
// of 2048 tokens over 30000, 32 query heads over 8: 887-901 us, 1160 TFLOP/s, a few calls after a pause (1.7 to 1.9 GHz);
// 1000-1060 us, 1000 TFLOP/s, call after call at the power limit.  A prompt of 8192 under a window of 4096: 353-374 and
// 394-416 us, 1130 and 1020 TFLOP/s.  P is rounded to the input type (the sum is of the unrounded weights): 0.0022
// of a bf16 output's norm, 0.0016 of which is the output's own rounding.  Measured and not kept: 16 worker warps, two to a row (1 to 4 % slower); one place
// for S and two for P (the same); the next S fetched into registers ahead (1.3 times as long).
// For pages the lengths are on the device, and every CTA finds its own share there: the items of all heads,
// laid end to end with their costs, are cut into as many equal stretches as there are CTAs.  An item
// that a border cuts is worked on in pieces along its keys; k_chunk_join puts them together in their order.
#include <cstring>
#include "zc_paged_groups.cuh"
#include "zc_layout.cuh"

namespace {

constexpr int kThreads = 384;
constexpr int kN = 64;                                // keys of a tile
constexpr int kTileLog2 = 6;
constexpr int kKvTile = kN * ZC_D * 2;                // 16 KB: [2][64][128 B]
constexpr int kKvBlock = kN * 128;
constexpr int kKS = 4, kVS = 5;                       // key and value buffers
constexpr uint32_t kCols = 512;                       // S_0 twice | S_1 twice | O_0 | O_1
constexpr int kOutTile = 32 * 64;                     // a warp's 32 rows x 32 channels on their way out
constexpr int kTiles = 2 * kTile + (kKS + kVS) * kKvTile + 8 * kOutTile;   // 224 KB
constexpr int kRingN = 2;                             // items fetched ahead
constexpr int kRingInts = 24;
constexpr int kSmem = kTiles + 1024 + 448 + 1024 + kRingN * kRingInts * 4;   // alignment, barriers, (m, sum) of group 1
constexpr float kTau = 3.f;                           // a new maximum is taken where it exceeds the old by this (base 2)
constexpr float kBigSum = 1024.f;                     // ... and looked for where a tile's weights sum to more than this
constexpr int kItemRows = 2 * kM;
// A piece's partial result: 32 x 256 groups of 4 channels, [group of channels][row], so that the threads that
// own neighbouring rows write neighbouring 16 bytes; then (maximum, sum) [row].
constexpr int kPartBytes = kItemRows * ZC_D * 4 + kItemRows * 8;
static_assert(kItemRows == ZC_CHUNK_PART_ROWS && kPartBytes == ZC_CHUNK_PART_BYTES, "as the joining kernel of groups reads them");
constexpr int kMaxItems = 13000;                      // items of a head, and requests, that a call may have: what the
                                                      // prologue keeps in the tiles' shared memory (16 bytes each)
constexpr int kMinPiece = 4;                          // tiles; a shorter piece goes to its neighbour

// Where a CTA's share begins: item `item` of all heads' (head * items + item of the head), key tile t of it.
struct Border { int item, t; };
// The item that the border before CTA c cuts, written by the first such CTA of the item.
struct ChunkJoin {
  int on, tok0, kv;
  int first, last;    // CTAs whose shares begin inside the item
  int row0, n;        // the request's first row, and its rows
  int pad;
};
struct ChunkWs {
  ChunkJoin* joins;   // [CTA]
  int* used;          // [CTA] its share is not empty
  char* parts;        // [CTA][2]: the piece at its share's start, the one at its end
};

// What a call is about: batch rows of dense tensors, requests' chunks in pages, or groups of requests whose rows all see
// the same first keys (no mask; every item's result is partial and joined with the rows' own keys elsewhere).
enum { kDense = 0, kPages = 1, kGroups = 2 };

struct ChunkArgs {
  ZcPagedArgs a;
  ChunkWs ws;
  ZcGroups gr;                         // kGroups
  long long o_req, o_row, o_head;      // elements: out; the log-sum-exp's are these / 128
  int tpt;                             // tokens per tile
  int l, items;                        // dense form: tokens per batch row, items per (batch row, KV head)
};

// A group's rows (those of its requests, which follow one another) and how many keys they share, as find_share has left it.
__device__ __forceinline__ Chunk load_group(const ChunkArgs& k, int g) {
  const ZcPagedArgs& a = k.a;
  Chunk c;
  c.p0 = k.gr.keys[g];
  const int r0 = group_border(a, k.gr, g), r1 = group_border(a, k.gr, g + 1);
  c.row0 = min(max(a.row_start[r0], 0), a.n_rows);
  c.n = c.p0 > 0 ? min(max(a.row_start[r1], 0), a.n_rows) - c.row0 : 0;
  return c;
}
__device__ __forceinline__ int item_tiles(const ZcPagedArgs& a, const Chunk& c, int tok0, int tpi) {
  const int last = min(tok0 + tpi, c.n) - 1;
  return zc_seen(c.p0 + tok0, c.p0 + last, a.window, a.sinks, kTileLog2).nb;
}

// Exclusive sum over the kThreads threads, and the total (a warp's values sum to less than 2^31).
__device__ __forceinline__ long long block_scan(int v, long long* s_warp, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  long long before = incl - v;
  *total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const long long u = s_warp[w];
    if (w < warp) before += u;
    *total += u;
  }
  return before;
}

// Cost of one of an item's tiles, and of the item.
__device__ __forceinline__ int item_width(int ntok, int tpt) { return ntok <= tpt ? kNarrowTile : kWideTile; }
__device__ __forceinline__ int item_cost(int nt, int width) { return nt * width + kItemCost; }
// The tile at which a border at `off` into an item's cost cuts it: 0 or nt where a piece would be short.
__device__ __forceinline__ int cut_tile(long long off, int nt, int width, int grain) {
  off -= kItemCost / 2;
  if (off <= 0) return 0;
  // (nt is below 2^24: beyond 31 bits the border lies behind the item)
  const int cost = (int)min(off, 0x7fffffffLL), t = (width == kWideTile ? cost / kWideTile : cost / kNarrowTile) & -grain;
  return t < kMinPiece ? 0 : nt - t < kMinPiece ? nt : t;
}

// Shares of fewer than eight tiles are cut at every fourth tile only: a piece of one or two costs more than they do (one
// chunk of 40 tokens, 32 heads over 8: over 1000 21.3 -> 19.0 us, over 4000 27.5 -> 23.6; shares of 25 tiles would lose 4 %).
__device__ __forceinline__ int cut_grain(long long all, int n_cta) { return all < 8LL * kWideTile * n_cta ? kMinPiece : 1; }

// This CTA's share of a paged call, found by the whole block in shared memory (16 bytes per request or item).
struct Share {
  Border begin, end;
  int items;          // of a head
  int r, in_req;      // the begin's request, and the item's number in it
  Chunk c;            // that request's (or group's) rows
  int lead;           // groups: the request through whose table
};
// What is found for all threads: the borders, and the item that the first of them lies in.
struct Found {
  Border border[2];
  long long start, all;   // the item's cost before it, and the cost of everything
  int nt, width, r, in_req, kv;   // (groups: kv is the first item's lead)
  Chunk c;
};
static_assert(sizeof(Found) <= 64, "it fits between the barriers and the sums");
template <int FORM>
__device__ __forceinline__ Share find_share(const ChunkArgs& k, char* scratch, long long* s_warp, Found* s_found,
                                            int n_cta) {
  const ZcPagedArgs& a = k.a;
  const int tid = threadIdx.x, tpi = 2 * k.tpt;
  const int n_req = FORM == kGroups ? k.gr.n : a.n_req;   // (groups take the requests' place below)
  // (the groups' tables have been made in front of the scratch)
  const GroupTables gt(scratch, k.gr.n, a.n_req);
  int* s_start = reinterpret_cast<int*>(scratch) + (FORM == kGroups ? GroupTables::kInts : 0);   // items before a request
  int* s_n = s_start + n_req + 1;
  int* s_p0 = s_n + n_req;
  int* s_cost = s_p0 + n_req;                          // cost of the head's items before an item
  int items = 0;
  for (int c0 = 0; c0 < n_req; c0 += kThreads) {
    const int r = c0 + tid;
    Chunk c;
    c.n = c.p0 = 0;
    if (r < n_req) {
      if (FORM == kGroups) {
        c.p0 = gt.keys[r];
        c.n = c.p0 > 0 ? gt.row[r + 1] - gt.row[r] : 0;
        k.gr.keys[r] = c.p0;   // (every CTA leaves the same where it reads it again)
        k.gr.lead[r] = gt.lead[r];
      } else {
        c = load_chunk(a, r);
      }
      s_n[r] = c.n;
      s_p0[r] = c.p0;
    }
    long long t;
    const long long at = block_scan((c.n + tpi - 1) / tpi, s_warp, &t);
    // (lengths that contradict the host's bounds cannot lead outside the scratch)
    const long long most = FORM == kGroups ? k.gr.most : kMaxItems;
    if (r < n_req) s_start[r] = (int)min(most, items + at);
    items = (int)min(most, items + t);
  }
  if (tid == 0) s_start[n_req] = items;
  __syncthreads();
  if (FORM == kGroups) {
    // what the joining kernel is to know of a request: its group's keys, its first row among the group's, the first item
    if (blockIdx.x == 0 && tid == 0) *k.gr.head = n_cta;
    for (int r = blockIdx.x + tid * n_cta; r < a.n_req; r += kThreads * n_cta) {
      const int g = gt.group_of(r);
      k.gr.info[r] = g < 0 ? make_int4(0, 0, 0, 0) : make_int4(gt.keys[g], max(0, gt.chunk(a, r).row0 - gt.row[g]), s_start[g], 0);
    }
  }
  auto request = [&](int i) {
    int lo = 0, hi = n_req;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (s_start[m] <= i) lo = m; else hi = m;
    }
    return lo;
  };
  auto tiles = [&](int i, int r, int* width) {
    const int tok0 = (i - s_start[r]) * tpi;
    Chunk c;
    c.row0 = 0;
    c.n = s_n[r];
    c.p0 = s_p0[r];
    *width = item_width(min(tpi, c.n - tok0), k.tpt);
    if (FORM == kGroups) return (c.p0 + kN - 1) >> kTileLog2;
    return item_tiles(a, c, tok0, tpi);
  };
  const int most = 0x7fffffff / max(items, 1);   // a head's cost stays in 31 bits
  long long head = 0;   // cost of a head
  for (int c0 = 0; c0 < items; c0 += kThreads) {
    const int i = c0 + tid;
    int cost = 0;
    if (i < items) {
      int width;
      const int nt = tiles(i, request(i), &width);
      cost = min(item_cost(nt, width), most);
    }
    long long t;
    const long long at = block_scan(cost, s_warp, &t);
    if (i < items) s_cost[i] = (int)(head + at);
    head += t;
  }
  if (tid == 0) s_cost[items] = (int)head;
  __syncthreads();
  // Borders before this CTA and the next (threads 0 and 1).
  const int c = blockIdx.x;
  const long long all = head * a.h_kv;
  if (tid < 2) {
    const long long at = zc_muldiv(c + tid, all, n_cta);
    Border b;
    b.item = items * a.h_kv;
    b.t = 0;
    Found f;
    f.start = f.all = all;
    f.nt = f.width = f.r = f.in_req = f.kv = 0;
    f.c.row0 = f.c.n = f.c.p0 = 0;
    if (at < all) {
      const int kv = all < (1 << 24) ? (int)((uint32_t)at / (uint32_t)head) : (int)(at / head);
      const long long in = at - kv * head;
      int lo = 0, hi = items;
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (s_cost[m] <= in) lo = m; else hi = m;
      }
      const int r = request(lo), nt = tiles(lo, r, &f.width), t = cut_tile(in - s_cost[lo], nt, f.width, cut_grain(all, n_cta));
      b.item = kv * items + lo;
      b.t = t;
      f.start = kv * head + s_cost[lo];
      f.nt = nt;
      f.r = r;
      f.in_req = lo - s_start[r];
      f.kv = kv;
      if (t > 0 && t == nt) {   // the next item
        b.item += 1;
        b.t = 0;
        const int next = lo + 1 < items ? lo + 1 : 0;
        f.r = request(next);
        f.in_req = next - s_start[f.r];
      }
      if (tid == 0) {
        if (FORM == kGroups) f.kv = gt.lead[f.r];
        f.c.n = s_n[f.r];
        f.c.p0 = s_p0[f.r];
        f.c.row0 = FORM == kGroups ? gt.row[f.r] : load_chunk(a, f.r).row0;
      }
    }
    s_found->border[tid] = b;
    if (tid == 0) {
      s_found->start = f.start;
      s_found->all = f.all;
      s_found->nt = f.nt;
      s_found->width = f.width;
      s_found->r = f.r;
      s_found->in_req = f.in_req;
      s_found->kv = f.kv;
      s_found->c = f.c;
    }
  }
  async_proxy_fence();   // the scratch's place is the tiles' from here on, whose copies come by the other proxy
  __syncthreads();
  Share s;
  s.begin = s_found->border[0];
  s.end = s_found->border[1];
  s.items = items;
  s.r = s_found->r;
  s.in_req = s_found->in_req;
  s.c = s_found->c;
  s.lead = s_found->kv;
  if (tid == kThreads - 1) {
    // (a thread that has nothing to do yet) what k_chunk_join is to know of the border before this CTA
    const Found f = *s_found;
    ChunkJoin j;
    j.on = 0;
    if (s.begin.t > 0) {
      // the CTAs around this one whose borders cut the same item
      auto cuts = [&](int d) {
        const int u = cut_tile(zc_muldiv(d, f.all, n_cta) - f.start, f.nt, f.width, cut_grain(f.all, n_cta));
        return u > 0 && u < f.nt;
      };
      j.first = j.last = c;
      while (j.first > 1 && cuts(j.first - 1)) --j.first;
      if (j.first == c) {
        while (j.last + 1 < n_cta && cuts(j.last + 1)) ++j.last;
        j.on = 1;
        if (FORM != kGroups) {
          const Chunk q = load_chunk(a, f.r);
          j.row0 = q.row0;
          j.n = q.n;
        }
        j.tok0 = f.in_req * tpi;
        j.kv = f.kv;   // (k_chunk_join's, which groups do without)
      }
    }
    k.ws.joins[c] = j;
    if (FORM == kGroups) k.gr.last[c] = j.on ? j.last : c;
    k.ws.used[c] = s.begin.item < s.end.item || s.begin.t < s.end.t;
  }
  return s;
}

// Shared-memory descriptor of a B operand whose N dimension is contiguous: rows are keys of 128 bytes
// (64 channels), groups of 8 rows 1024 bytes apart, the other 64 channels one k-block further.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(kKvBlock >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// The tensor cores take a few products ahead of the one they work on and no more, so what the issuing
// thread does between two of them is time lost: descriptors of whole tiles are made beforehand and a step
// adds a constant to each (the address field counts 16 bytes and cannot overflow into its neighbour).
__device__ __forceinline__ void mma_s(uint32_t tmem_s, uint64_t da, uint64_t db, uint32_t idesc) {
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const uint64_t qo = (uint64_t)(((ks >> 2) * kKBlock + (ks & 3) * 32) >> 4);
    const uint64_t ko = (uint64_t)(((ks >> 2) * kKvBlock + (ks & 3) * 32) >> 4);
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_s),
        "l"(da + qo), "l"(db + ko), "r"(idesc), "r"(ks > 0 ? 1u : 0u)
        : "memory");
  }
}
// O (+)= P V: four steps of 16 keys (A = P from tensor memory, 8 columns a step).
__device__ __forceinline__ void mma_pv(uint32_t tmem_o, uint32_t tmem_p, uint64_t db, uint32_t idesc, bool accumulate) {
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_o),
        "r"(tmem_p + 8u * ks), "l"(db + (uint64_t)((ks * 16 * 128) >> 4)), "r"(idesc), "r"((accumulate || ks > 0) ? 1u : 0u)
        : "memory");
}
// An item as the fetching warp hands it to the other roles.
struct Item {
  int r, kv, tok0, ntok;      // request (dense form: batch row), KV head, tokens; r < 0: no more items
  int row0;                   // row of the request's token 0
  int p_first, t0, t1, slot;
  int narrow;                 // one tile of rows: the groups take the even and the odd key tiles
  ZcSeen s;
  int ga[2], ge[2];           // key tiles from .. to that group 0 / 1 takes part in (narrow: both all)
  __device__ __forceinline__ int key0(int t) const { return (t < s.nsb ? t : s.wb0 + t - s.nsb) << kTileLog2; }
};
static_assert(sizeof(Item) <= kRingInts * 4, "an item fits its place in the ring");

// Item of a dense call.
__device__ __forceinline__ Item dense_item(const ChunkArgs& k, long long idx) {
  const ZcPagedArgs& a = k.a;
  const int units = a.n_req * a.h_kv, q = (int)(idx / units), unit = (int)(idx - (long long)q * units);
  Item it;
  it.r = unit / a.h_kv;
  it.kv = unit - it.r * a.h_kv;
  it.tok0 = (k.items - 1 - q) * 2 * k.tpt;   // the last, longest rows first
  it.slot = -1;
  it.row0 = 0;
  it.p_first = it.tok0;
  it.t0 = 0;
  it.t1 = 1 << 30;
  return it;
}

// Fills in what follows from the rows (n tokens in the request) and the first and last key tile asked for.
__device__ __forceinline__ void finish_item(const ChunkArgs& k, int n, Item& it) {
  const ZcPagedArgs& a = k.a;
  const int tpi = 2 * k.tpt;
  it.ntok = min(tpi, n - it.tok0);
  it.narrow = it.ntok <= k.tpt;
  it.s = zc_seen(it.p_first, it.p_first + it.ntok - 1, a.window, a.sinks, kTileLog2);
  it.t1 = min(it.t1, it.s.nb);
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int first = it.p_first + g * k.tpt, last = it.p_first + min(it.ntok, (g + 1) * k.tpt) - 1;
    const int lo = max(0, first - a.window + 1), hi = max(0, last + 1);
    const int end = it.s.nsb + max(0, ((hi + kN - 1) >> kTileLog2) - it.s.wb0);
    // sinks: from the first tile on, also where the other group's window still reaches back to them
    const int begin = a.sinks > 0 ? 0 : max(0, (lo >> kTileLog2) - it.s.wb0);
    it.ga[g] = it.narrow ? it.t0 : max(it.t0, begin);
    it.ge[g] = it.narrow ? it.t1 : min(it.t1, end);
  }
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// The weights of 64 keys, 2^(v * scale - m), packed to the input type; returns their sum (of the unrounded
// values).  Rounded once, also in a group's item, whose rows would have two parts as single tokens: with the rest as a second
// part (twice the products of O) the error against 64 bits is the output's own, bf16 0.0017 of its norm instead of 0.0023, and
// the calls take 13 to 18 % longer (64 requests on 8192: 42 -> 49 us, 128 on 30000: 93 -> 107).
// All exponentials go through the exp2 unit: a quarter of them by a polynomial on the FMA pipe
// instead measured the same to 7 % slower.
template <typename T> __device__ __forceinline__ float weights(const float* v, float scale, float m, uint32_t* w) {
  const float2 sc = make_float2(scale, scale), neg_m = make_float2(-m, -m);
  float2 add[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < kN / 2; ++c) {
    const float2 x = fma2(make_float2(v[2 * c], v[2 * c + 1]), sc, neg_m);
    const float2 p = make_float2(zc_exp2(x.x), zc_exp2(x.y));
    add[c & 1] = add2(add[c & 1], p);
    w[c] = pack2<T>(p.x, p.y);
  }
  add[0] = add2(add[0], add[1]);
  return add[0].x + add[0].y;
}

// The same for a group's item: all rows see all of its keys.
__device__ __forceinline__ void finish_group_item(const ChunkArgs& k, const Chunk& c, Item& it) {
  it.ntok = min(2 * k.tpt, c.n - it.tok0);
  it.narrow = it.ntok <= k.tpt;
  it.s.lo = it.s.sink_n = it.s.nsb = it.s.wb0 = 0;
  it.s.hi = c.p0;
  it.s.nb = (c.p0 + kN - 1) >> kTileLog2;
  it.t1 = min(it.t1, it.s.nb);
  it.ga[0] = it.ga[1] = it.t0;
  it.ge[0] = it.ge[1] = it.t1;
}

// Bits 0 .. n - 1 of 64.
__device__ __forceinline__ uint64_t below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
template <typename T, int FORM>
__global__ void __launch_bounds__(kThreads, 1)
    k_chunk_attention(const ChunkArgs k, const __grid_constant__ CUtensorMap qmap,
                      const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  constexpr bool PAGED = FORM != kDense;
  const ZcPagedArgs& a = k.a;
  const uint32_t raw_u = zc_smem_u32(smem_raw);
  const uint32_t base_u = (raw_u + 1023u) & ~1023u;
  char* base = smem_raw + (base_u - raw_u);
  const uint32_t q_addr = base_u, k_addr = base_u + 2 * kTile, v_addr = k_addr + kKS * kKvTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + kTiles);
  uint64_t* q_full = bars;                  // [3] Q of a wide item's group 0 landed, of its group 1, of a narrow item
  uint64_t* q_free = bars + 3;              // group 1's last S of a narrow item completed
  uint64_t* k_full = bars + 4;              // [kKS] key tile landed
  uint64_t* k_free = k_full + kKS;          // [kKS] both groups are through with that tile
  uint64_t* v_full = k_free + kKS;          // [kVS] value tile landed
  uint64_t* v_free = v_full + kVS;          // [kVS] both groups are through with that tile
  uint64_t* s_done = v_free + kVS;          // [2][2] S_g of a tile completed, by its place
  uint64_t* p_full = s_done + 4;            // [2][2] the group's four warps have written P_g
  uint64_t* o_last = p_full + 4;            // [2] the group's last P V but one of an item completed
  uint64_t* o_done = o_last + 2;            // [2] the group's last P V of an item completed
  uint64_t* i_full = o_done + 2;            // [kRingN] an item is in the ring
  uint64_t* i_free = i_full + kRingN;       // [kRingN] all roles have read it
  uint64_t* m_free = i_free + kRingN;       // [2] the groups' meeting over a narrow item is over (in turn)
  uint64_t* meet_bar = m_free + 2;          // the groups' eight warps meet over a narrow item
  uint64_t* drained = meet_bar + 1;         // [2] all products of the group completed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 2);
  uint32_t* meet_slot = tmem_slot + 1;      // meetings that all eight warps have come to; ~0: there are no more
  float2* s_ms = reinterpret_cast<float2*>(base + kTiles + 448);                    // [128] narrow items: group 1's (m, sum)
  int* ring = reinterpret_cast<int*>(base + kTiles + 448 + 1024);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int n_cta = gridDim.x;
  if (FORM == kGroups) {
    // The kernel behind this one, of the requests' own keys, does not wait for it: it takes the CTAs that are not needed
    // here.  So it may start only once what came before both is complete.
    zc_wait_for_last();
    zc_let_next_start();
    n_cta = plan_groups<kThreads>(a, k.gr, GroupTables(base, k.gr.n, a.n_req), k.tpt, gridDim.x);
    if (blockIdx.x == 0 && tid == 0) *reinterpret_cast<volatile int*>(k.gr.told) = 1 + n_cta;
    if (n_cta == 0)
      for (int r = blockIdx.x + tid * gridDim.x; r < a.n_req; r += kThreads * gridDim.x) k.gr.info[r] = make_int4(0, 0, 0, 0);
    if ((int)blockIdx.x >= n_cta) return;
  } else {
    zc_let_next_start();
  }
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) bar_init(&q_full[i], 1);   // q_free too
    bar_init(&m_free[0], 1);
    bar_init(&m_free[1], 1);
    bar_init(meet_bar, 8);
    *meet_slot = 0;
    for (int i = 0; i < kKS; ++i) {
      bar_init(&k_full[i], 1);
      bar_init(&k_free[i], 2);
    }
    for (int i = 0; i < kVS; ++i) {
      bar_init(&v_full[i], 1);
      bar_init(&v_free[i], 2);
    }
    for (int g = 0; g < 2; ++g) {
      for (int i = 0; i < 2; ++i) {
        bar_init(&s_done[2 * g + i], 1);
        bar_init(&p_full[2 * g + i], 4);
      }
      bar_init(&o_last[g], 1);
      bar_init(&o_done[g], 1);
      bar_init(&drained[g], 1);
    }
    for (int i = 0; i < kRingN; ++i) {
      bar_init(&i_full[i], 1);
      bar_init(&i_free[i], 11);   // K, two warps for the products, eight worker warps
    }
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  if (warp == 0) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(zc_smem_u32(tmem_slot)),
                 "r"(kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  if (FORM != kGroups) zc_wait_for_last();
  Share share;
  if (PAGED) share = find_share<FORM>(k, base, reinterpret_cast<long long*>(s_ms), reinterpret_cast<Found*>(base + kTiles + 384), n_cta);

  uint32_t n_item = 0;   // items taken from the ring
  // Next item of the ring; a whole warp calls.  False: there are no more (or a wait ran out).
  auto next_item = [&](Item& it) {
    const uint32_t at = n_item % kRingN;
    if (!warp_wait(&i_full[at], (n_item / kRingN) & 1u)) return false;
    const int* src = ring + at * kRingInts;
    int* dst = reinterpret_cast<int*>(&it);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Item) / 4); ++i) dst[i] = src[i];
    __syncwarp();
    if (lane == 0) bar_arrive(&i_free[at]);
    ++n_item;
    return it.r >= 0;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
    // The key (or value) tiles of an item through their ring; the whole warp calls.  False: a wait ran out.
    uint32_t stage = 0, phase = 1;   // of this warp's stream; the first wait for a free place succeeds at once
    auto stream = [&](const Item& it, const CUtensorMap* map, uint32_t at, uint64_t* full, uint64_t* free, uint32_t places) {
      const int rows = PAGED ? min(kN, 1 << a.page_log2) : kN;
      // page ids: lane i holds that of page base + i, and of the 32 pages behind those
      int base = -64, now = -1, next = -1;
      auto table_at = [&](int page) { return page < a.table_width ? a.table[(long long)it.r * a.table_width + page] : -1; };
#pragma unroll 1
      for (int t = it.t0; t < it.t1; ++t) {
        const int key0 = it.key0(t);
        int page = it.r, row = key0;   // dense form: a batch row is a page
        bool on = lane == 0;
        uint32_t bytes = kKvTile;
        if (PAGED) {
          const int page0 = key0 >> a.page_log2, b = page0 & ~31;
          if (b != base) {
            now = b == base + 32 ? next : table_at(b + lane);
            next = table_at(b + 32 + lane);
            base = b;
          }
          const int id = __shfl_sync(0xffffffffu, now, (page0 + lane) & 31);
          page = id >= 0 && id < a.n_pages ? id : a.n_pages;   // beyond the pool: arrives as zeros
          row = key0 & ((1 << a.page_log2) - 1);
          if (rows < kN) {
            // lane i brings the i-th page of the tile, if any row of the item sees a key of it
            const int pk0 = key0 + lane * rows;
            on = lane < kN / rows && (pk0 < it.s.sink_n || (pk0 < it.s.hi && pk0 + rows > it.s.lo));
            bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, on)) * (uint32_t)rows * (ZC_D * 2);
          }
        }
        if (!warp_wait(&free[stage], phase)) return false;
        if (lane == 0) expect_bytes(&full[stage], bytes);
        __syncwarp();
        if (on) {
          const uint32_t dst = at + stage * kKvTile + lane * rows * 128;
          page_copy(map, dst, &full[stage], row, 0, it.kv, page);
          if (rows < kN) page_copy(map, dst + kKvBlock, &full[stage], row, 1, it.kv, page);
        }
        __syncwarp();
        if (++stage == places) {
          stage = 0;
          phase ^= 1u;
        }
      }
      return true;
    };
    // The places before `stage` were filled in this round of the ring, the others in the one before (or never).
    auto landed = [&](uint64_t* full, uint32_t places) {
      for (uint32_t i = 0; i < places; ++i) drain(&full[i], i < stage ? phase ^ 1u : phase);
    };
    if (warp == 2) {
      // ---- items, and V ----
      // Dense form: the items longest first, every other round of the CTAs backwards, so that each gets about the
      // same sum (a causal prompt of 8192: 486 us in rounds all one way, 444 us so; window of 4096: 369 -> 347 us).
      const long long n_idx = (long long)k.items * a.n_req * a.h_kv;
      long long idx = blockIdx.x, round = 0;
      bool back = false;
      Border at = share.begin;
      int r = share.r, in_req = share.in_req, lead = share.lead;
      Chunk c;
      c.row0 = c.n = c.p0 = 0;
      auto load = [&](int i) { return FORM == kGroups ? load_group(k, i) : load_chunk(a, i); };
      if (PAGED && share.items > 0) c = share.c;
      auto find_item = [&](Item& it) {   // the share's next item; r < 0: there is none
        it.r = -1;
        if (!PAGED) {
          if (idx < n_idx) {
            it = dense_item(k, idx);
            finish_item(k, k.l, it);
            round += gridDim.x;
            back = !back;
            idx = round + (back ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
          }
          return;
        }
        if (at.item > share.end.item || (at.item == share.end.item && at.t >= share.end.t)) return;
        // (only the share's first item can begin, and only its last can end, inside)
        it.r = FORM == kGroups ? lead : r;   // whose table has the item's pages
        it.kv = at.item / share.items;
        it.tok0 = in_req * 2 * k.tpt;
        it.row0 = c.row0;
        it.p_first = c.p0 + it.tok0;
        it.t0 = at.t;
        it.t1 = at.item == share.end.item ? share.end.t : 1 << 30;
        if (FORM == kGroups) finish_group_item(k, c, it);
        else finish_item(k, c.n, it);
        it.slot = it.t0 > 0 ? 2 * (int)blockIdx.x : it.t1 < it.s.nb ? 2 * (int)blockIdx.x + 1 : -1;
        // where the item's result will be: with its rows, or in pieces from the next CTA's border on
        if (FORM == kGroups && it.t0 == 0 && lane == 0)
          k.gr.cut[(long long)(at.item - it.kv * share.items) * a.h_kv + it.kv] = it.slot >= 0 ? (int)blockIdx.x + 1 : 0;
        ++at.item;
        at.t = 0;
        if (at.item > share.end.item || (at.item == share.end.item && share.end.t == 0)) return;
        if ((++in_req) * 2 * k.tpt >= c.n) {
          // the next request with rows (after the last one's, the next head's first), 32 at a time
          in_req = 0;
          const int n_req = FORM == kGroups ? k.gr.n : a.n_req;
          for (int r0 = at.item % share.items == 0 ? 0 : r + 1; r0 < n_req; r0 += 32) {
            Chunk x;
            x.row0 = x.n = x.p0 = 0;
            if (r0 + lane < n_req) x = load(r0 + lane);
            const unsigned some = __ballot_sync(0xffffffffu, x.n > 0);
            if (some) {
              const int src = __ffs(some) - 1;
              r = r0 + src;
              if (FORM == kGroups) lead = k.gr.lead[r];
              c.row0 = __shfl_sync(0xffffffffu, x.row0, src);
              c.n = __shfl_sync(0xffffffffu, x.n, src);
              c.p0 = __shfl_sync(0xffffffffu, x.p0, src);
              break;
            }
          }
        }
      };
      uint32_t n = 0;   // items announced
      auto announce = [&](const Item& it) {
        const uint32_t place = n % kRingN;
        if (n >= kRingN && !warp_wait(&i_free[place], (n / kRingN - 1) & 1u)) return false;
        if (lane == 0) {
          int* dst = ring + place * kRingInts;
          const int* src = reinterpret_cast<const int*>(&it);
#pragma unroll
          for (int i = 0; i < (int)(sizeof(Item) / 4); ++i) dst[i] = src[i];
          bar_arrive(&i_full[place]);
        }
        __syncwarp();
        ++n;
        return true;
      };
      Item it, then;
      find_item(it);
      bool ok = announce(it);
      while (ok && it.r >= 0) {
        find_item(then);
        ok = announce(then) && stream(it, &vmap, v_addr, v_full, v_free, kVS);
        it = then;
      }
      landed(v_full, kVS);
    } else if (warp == 1) {
      // ---- K ----
      uint32_t meetings = 0, met = 0;   // narrow items with tiles, meetings of them waited for
      bool ok = true;
      Item it;
      while (ok && next_item(it)) {
        if (it.t0 >= it.t1) continue;
        // a wide item's second Q tile goes where the groups meet over narrow ones
        for (; ok && met + (it.narrow ? 1u : 0u) < meetings; ++met) ok = warp_wait(&m_free[met & 1u], (met >> 1) & 1u);
        meetings += it.narrow ? 1u : 0u;
        ok = ok && stream(it, &kmap, k_addr, k_full, k_free, kKS);
      }
      landed(k_full, kKS);
    } else {
      // ---- matrix products of group g ----
      // Per tile: O += P V, then the group's S two of its tiles on, into the place that this P leaves.  Each
      // group has a warp of its own for them: the tensor cores queue only a few products, and what one warp
      // spends on barriers and commits the other's products fill.
      const int g = uniform(warp == 0 ? 0 : 1);
      const uint32_t tm = (uint32_t)uniform((int)tmem), tm_s = tm + g * kM, tm_o = tm + (2 + g) * kM;
      const uint32_t idesc_s = (instr_desc<T>() & ~(0x3Fu << 17)) | ((uint32_t)(kN >> 3) << 17);
      const uint32_t idesc_pv = instr_desc<T>() | (1u << 16);   // B with its N dimension contiguous
      const uint64_t q_desc = smem_desc(q_addr), k_desc = smem_desc(k_addr), v_desc = desc_mn(v_addr);
      uint32_t n_s = 0, n_p = 0;                           // tiles of the group whose S / P V is issued
      uint32_t n_wide = 0, n_narrow = 0; // wide and narrow items so far
      bool met = false;                                    // the item before was a narrow one
      uint32_t ks = 0, kp = 0, vs = 0, vp = 0;             // place and phase of the next key and value tile
      uint64_t* q_last = nullptr;                          // barrier and phase of the last Q copy issued
      uint32_t q_last_phase = 0;
      bool ok = true;                                      // no wait has run out
      Item it;
      while (ok && next_item(it)) {
        const int t0 = uniform(it.t0), n = uniform(it.t1) - t0, narrow = uniform(it.narrow);
        const int ga = uniform(g ? it.ga[1] : it.ga[0]) - t0, ge = uniform(g ? it.ge[1] : it.ge[0]) - t0;
        if (n <= 0) continue;
        const int ahead = narrow ? 4 : 2, step = narrow ? 2 : 1;
        const uint64_t qd = q_desc + (uint64_t)((narrow ? 0 : g) * (kTile >> 4));
        auto mine = [&](int i) { return narrow ? (i & 1) == g : i >= ga && i < ge; };
        auto keys = [&](int i) {        // the item's key tile i: its S, and the tile's release
          ok = warp_wait(&k_full[ks], kp);
          if (!ok) return;
          const uint64_t kd = k_desc + (uint64_t)(ks * (kKvTile >> 4));
          const uint32_t place = n_s & 1u;
          const bool on = mine(i);
          if (elect_one()) {
            if (on) {
              mma_s(tm_s + place * kN, qd, kd, idesc_s);
              mma_commit(&s_done[2 * g + place]);
            }
            mma_commit(&k_free[ks]);
            if (i + 1 == n && narrow && g == 1) mma_commit(q_free);
          }
          __syncwarp();
          n_s += on ? 1u : 0u;
          if (++ks == kKS) {
            ks = 0;
            kp ^= 1u;
          }
        };
        // Q of the group's rows, brought by the warp that multiplies it: the products that read the place are through
        // (each S has come back as P), but those of group 1 with a narrow item's rows, which both groups read.  Where
        // group 1's tile goes the groups may be meeting still: not once the item's first key tile is there.
        uint64_t* q_bar = &q_full[narrow ? 2 : g];
        const uint32_t q_phase = (narrow ? n_narrow : n_wide) & 1u;
        if (!narrow || g == 0) {
          if (met) ok = g == 0 ? warp_wait(q_free, (n_narrow - 1) & 1u) : warp_wait(&k_full[ks], kp);
          if (!ok) break;
          q_last = q_bar;
          q_last_phase = q_phase;
          if (elect_one()) {
            expect_bytes(q_bar, (uint32_t)(k.tpt * a.G * ZC_D * 2));
            for (int kb = 0; kb < 2; ++kb)
              q_copy(&qmap, q_addr + g * kTile + kb * kKBlock, q_bar, kb, it.kv * a.G, it.row0 + it.tok0 + g * k.tpt,
                     PAGED ? 0 : it.r);
          }
          __syncwarp();
        }
        ok = warp_wait(q_bar, q_phase);
        if (narrow) ++n_narrow; else ++n_wide;
        met = narrow;
#pragma unroll 1
        for (int i = 0; ok && i < min(n, ahead); ++i) keys(i);
#pragma unroll 1
        for (int i = 0; ok && i < n; ++i) {
          // Tiles in the midst of a wide item, the same work with nothing to decide: what this warp does beside its
          // products is what a step takes longer than they do.
          if (!narrow && i == ga + 1) {
            const int mid_end = min(ge - 2, n - 3);
#pragma unroll 1
            for (; i < mid_end; ++i) {
              const uint32_t place = n_p & 1u;
              const uint64_t vd = v_desc + (uint64_t)(vs * (kKvTile >> 4)), kd = k_desc + (uint64_t)(ks * (kKvTile >> 4));
              uint64_t *kf = &k_full[ks], *vf = &v_full[vs], *pf = &p_full[2 * g + place];
              const bool k_in = bar_try(kf, kp) || bar_wait(kf, kp), v_in = bar_try(vf, vp) || bar_wait(vf, vp);
              const bool p_in = bar_try(pf, (n_p >> 1) & 1u) || bar_wait(pf, (n_p >> 1) & 1u);
              const bool in = k_in && v_in && p_in;
              tc_fence_after();
              if (elect_one() && in) {
                mma_pv(tm_o, tm_s + place * kN, vd, idesc_pv, true);
                mma_commit(vf + kVS);    // v_free
                mma_s(tm_s + place * kN, qd, kd, idesc_s);
                mma_commit(&s_done[2 * g + place]);
                mma_commit(kf + kKS);    // k_free
              }
              __syncwarp();
              ++n_p;
              ++n_s;
              const bool kw = ks + 1 == kKS, vw = vs + 1 == kVS;
              ks = kw ? 0 : ks + 1;
              vs = vw ? 0 : vs + 1;
              kp ^= kw ? 1u : 0u;
              vp ^= vw ? 1u : 0u;
              ok = __all_sync(0xffffffffu, in);   // (behind the products: nothing waits for the vote)
              if (!ok) break;
            }
            if (!ok || i >= n) break;
          }
          ok = warp_wait(&v_full[vs], vp);
          if (!ok) break;
          const uint64_t vd = v_desc + (uint64_t)(vs * (kKvTile >> 4));
          const bool on = mine(i);
          if (on) {
            const uint32_t place = n_p & 1u;
            const bool first = narrow ? i < 2 : i == ga;
            const bool last = narrow ? i + step >= n : i + 1 == ge;
            const bool last_but_one = !last && (narrow ? i + 2 * step >= n : i + 2 == ge);
            ok = warp_wait(&p_full[2 * g + place], (n_p >> 1) & 1u);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              mma_pv(tm_o, tm_s + place * kN, vd, idesc_pv, !first);
              mma_commit(&v_free[vs]);
              if (last_but_one) mma_commit(&o_last[g]);
              if (last) mma_commit(&o_done[g]);
            }
            ++n_p;
          } else if (elect_one()) {
            mma_commit(&v_free[vs]);
          }
          __syncwarp();
          if (++vs == kVS) {
            vs = 0;
            vp ^= 1u;
          }
          if (i + ahead < n) keys(i + ahead);
        }
      }
      if (q_last) drain(q_last, q_last_phase);
      if (n_s > 0) {
        if (elect_one()) mma_commit(&drained[g]);
        __syncwarp();
        drain(&drained[g], 0);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;\n");
    const int g = (warp >> 2) - 1, quarter = warp & 3, row = quarter * 32 + lane;
    const int tok_in = row / a.G, head_in = row - tok_in * a.G;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t tmem_g = tmem + lane_off + (uint32_t)g * kM, tmem_o = tmem + lane_off + (uint32_t)(2 + g) * kM;
    const float scale = kLog2e * rsqrtf((float)ZC_D);
    uint32_t tile0 = 0, n_s = 0, n_o = 0, n_last = 0, meetings = 0;
    // Both groups meet over a narrow item: a hardware barrier, which cannot be given up.  So they first agree that all
    // eight warps are here: whoever settles the count first, by the bounded wait's success or by its end, settles it for
    // all (a warp that left, or whose wait ran out, is never waited for; ~0 stays).
    auto groups_sync = [&]() { asm volatile("bar.sync 1, 256;\n" ::: "memory"); };
    auto all_here = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(meet_bar);
      const bool here = bar_wait(meet_bar, meetings & 1u);
      uint32_t to = here ? meetings + 1u : ~0u;
      if (lane == 0) {
        const uint32_t was = atomicCAS(meet_slot, meetings, to);
        if (was != meetings) to = was;
      }
      return __shfl_sync(0xffffffffu, to, 0) == meetings + 1u;
    };
    Item it;
    while (next_item(it)) {
      const int rows_at = it.narrow ? 0 : g;                         // which tile of rows
      const int tok = rows_at * k.tpt + tok_in;                      // token of the item
      const bool valid = tok_in < k.tpt && tok < it.ntok;
      const int pos = valid ? (FORM == kGroups ? it.s.hi - 1 : it.p_first + tok) : -1;   // (all of a group's see all its keys)
      const int first = it.p_first + rows_at * k.tpt;
      const int last = it.p_first + min(it.ntok, (rows_at + 1) * k.tpt) - 1;
      const int ga = g ? it.ga[1] : it.ga[0], ge = g ? it.ge[1] : it.ge[0];
      const int step = it.narrow ? 2 : 1, t_first = it.narrow ? it.t0 + g : ga;
      float m_run = kNoMax, s_run = 0.f;
      bool unset = true;     // a row of the warp has seen no key yet, or has its maximum beyond kFarMax
      for (int t = t_first; t < ge; t += step) {
        const int key0 = it.key0(t);
        const uint32_t place = n_s & 1u, tmem_s = tmem_g + place * kN;
        float v[kN];
        bar_wait(&s_done[2 * g + place], (n_s >> 1) & 1u);
        ++n_s;
        tc_fence_after();
#pragma unroll
        for (int h = 0; h < 2; ++h) tmem_ld32_nowait(v + 32 * h, tmem_s + 32 * h);
#pragma unroll
        for (int h = 0; h < 2; ++h) tmem_wait32(v + 32 * h);
        const bool edge = FORM == kGroups ? key0 + kN > it.s.hi
                                          : key0 + kN - 1 > first || (key0 <= last - a.window && key0 + kN > a.sinks);
        if (edge) {
          // the tile crosses the diagonal, the window's edge or the end of the sinks
          const uint64_t seen = below(pos + 1 - key0) & (~below(pos + 1 - a.window - key0) | below(a.sinks - key0));
          const uint32_t seen2[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
#pragma unroll
          for (int e = 0; e < kN; ++e)
            if (!((seen2[e >> 5] >> (e & 31)) & 1u)) v[e] = -INFINITY;
          // values that no row of the item sees may hold anything (a weight of 0 times NaN is NaN)
          if (key0 + kN > it.s.hi || (key0 < it.s.lo && key0 + kN > it.s.sink_n)) {
            const uint32_t tile = tile0 + (uint32_t)(t - it.t0), vs = tile % kVS;
            bar_wait(&v_full[vs], (tile / kVS) & 1u);
            const int key = key0 + (row & (kN - 1));               // a thread clears 64 of a key's channels
            if (key >= it.s.hi || (key < it.s.lo && key >= it.s.sink_n)) {
              char* at = base + (v_addr - base_u) + vs * kKvTile + (row / kN) * kKvBlock + (row & (kN - 1)) * 128;
#pragma unroll
              for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(at + c * 16) = make_uint4(0, 0, 0, 0);
            }
            async_proxy_fence();
          }
        }
        // With the maximum that the row has so far, which as a rule is near enough: no pass over the logits for a
        // new one.  The sum tells where it is not (a weight above 2^4 at least, 2^10 at most stays unseen).  Only the
        // item's rows have a say: the tile's other rows hold another request's queries or what was there before, and
        // a new maximum changes how the weights round.
        uint32_t w[kN / 2];
        float sum = 0.f;
        bool renew = edge || unset;
        if (!renew) {
          sum = weights<T>(v, scale, m_run, w);
          renew = __any_sync(0xffffffffu, valid && !(sum <= kBigSum));
        }
        if (renew) {
          float mx4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int e = 4; e < kN; e += 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx4[i] = e + 4 < kN ? max3(mx4[i], v[e + i], v[e + 4 + i]) : fmaxf(mx4[i], v[e + i]);
          const float top = fmaxf(max3(mx4[0], mx4[1], mx4[2]), mx4[3]), mx = top * scale;
          const bool grow = valid && mx > m_run + kTau;
          if (__any_sync(0xffffffffu, grow)) {
            const float alpha = grow ? zc_exp2(m_run - mx) : 1.f;
            if (t > t_first) {
              // O has every product up to the tile before once the next tile's S is there (it was issued behind
              // them), or, at the last tile, once they say so themselves
              if (t + step < ge) bar_wait(&s_done[2 * g + (n_s & 1u)], (n_s >> 1) & 1u);
              else bar_wait(&o_last[g], n_last & 1u);
              tc_fence_after();
#pragma unroll 1
              for (int q8 = 0; q8 < 16; ++q8) {
                float o[8];
                tmem_ld8(o, tmem_o + 8 * q8);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] *= alpha;
                tmem_st8(o, tmem_o + 8 * q8);
              }
            }
            s_run *= alpha;
            if (grow) m_run = mx;
          }
          unset = __any_sync(0xffffffffu, valid && !(fabsf(m_run) < kFarMax));
          float less = m_run;
          if (unset && __any_sync(0xffffffffu, valid && !(fabsf(m_run) < kFarMax) && m_run != kNoMax)) {
            // the maximum's q.k waits where outputs leave from
            if (valid && !(fabsf(m_run) < kFarMax) && m_run != kNoMax) {
              float* keep = reinterpret_cast<float*>(base + 2 * kTile + (kKS + kVS) * kKvTile + (warp - 4) * kOutTile) + lane;
              if (grow) *keep = top;
#pragma unroll
              for (int e = 0; e < kN; ++e) v[e] -= *keep;
              less = 0.f;
            }
          }
          sum = weights<T>(v, scale, less, w);
        }
        tmem_st32(w, tmem_s);
        asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(&p_full[2 * g + place]);
        s_run += sum;
      }
      if (ge - t_first > step) ++n_last;   // an item of two or more of this group's tiles
      tile0 += (uint32_t)max(0, it.t1 - it.t0);
      // ---- the row's output and log-sum-exp, or its partial result ----
      const bool any = t_first < ge;
      if (any) {
        bar_wait(&o_done[g], n_o & 1u);
        ++n_o;
        tc_fence_after();
      }
      bool meet = it.narrow && it.t0 < it.t1;
      float f_own = 1.f, f_other = 0.f;
      if (meet && g == 1) s_ms[row] = make_float2(m_run, s_run);
      if (meet) meet = all_here();
      const bool other = meet && it.t0 + 1 < it.t1;                  // group 1 has a share of a narrow item
      if (meet) {
        // group 1's sums, and its O by halves, to group 0
        if (g == 0 && other) {
          const float2 o = s_ms[row];
          const float m = fmaxf(m_run, o.x);
          f_own = zc_exp2(m_run - m);
          f_other = zc_exp2(o.x - m);
          s_run = s_run * f_own + o.y * f_other;
          m_run = m;
        }
      }
      const bool writer = valid && !(it.narrow && g == 1);
      const bool some = any && s_run > 0.f;
      const float inv = some ? 1.f / s_run : 0.f;
      const int h = it.kv * a.G + head_in;
      const long long at = (PAGED ? 0 : it.r * k.o_req) + (long long)(it.row0 + it.tok0 + tok) * k.o_row + h * k.o_head;
      char* part = PAGED && it.slot >= 0 ? k.ws.parts + (long long)it.slot * kPartBytes : nullptr;
      float* whole = FORM == kGroups ? k.gr.rows + at / ZC_D * ZC_PART_STRIDE : nullptr;   // (maximum, sum, -, -, 128 sums)
      const int prow = rows_at * kM + row;
      // Output rows leave through the warp's 2 KB of shared memory, 32 channels at a time, so that a store writes 64
      // bytes of each of eight rows: lane i then has rows i / 4 + 8 j, whose places it asks the owners for.
      const unsigned writers = __ballot_sync(0xffffffffu, writer);
      long long at_j[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) at_j[j] = __shfl_sync(0xffffffffu, at, (lane >> 2) + 8 * j);
      char* stage = base + 2 * kTile + (kKS + kVS) * kKvTile + (warp - 4) * kOutTile;
#pragma unroll 1
      for (int q4 = 0; q4 < 4; ++q4) {
        float o[32];
        if (any) {
          tmem_ld32_nowait(o, tmem_o + 32 * q4);
          tmem_wait32(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (other) {
          // through the place of the second Q tile: 128 rows x 32 channels, twice
          float4* xr = reinterpret_cast<float4*>(base + kTile) + row * 16 + 8 * (q4 & 1);
          if (g == 1) {
#pragma unroll
            for (int c = 0; c < 8; ++c) xr[c ^ (row & 7)] = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
            async_proxy_fence();
          }
          groups_sync();   // (group 0 has read the half before last by now)
          if (g == 0) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float4 x = xr[c ^ (row & 7)];
              o[4 * c] = o[4 * c] * f_own + x.x * f_other;
              o[4 * c + 1] = o[4 * c + 1] * f_own + x.y * f_other;
              o[4 * c + 2] = o[4 * c + 2] * f_own + x.z * f_other;
              o[4 * c + 3] = o[4 * c + 3] * f_own + x.w * f_other;
            }
          }
        }
        if (part) {
          if (writer)
#pragma unroll
            for (int c = 0; c < 8; ++c)
              reinterpret_cast<float4*>(part)[(8 * q4 + c) * kItemRows + prow] =
                  make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
        } else if (FORM == kGroups) {
          if (writer)
#pragma unroll
            for (int c = 0; c < 8; ++c)
              *reinterpret_cast<float4*>(whole + 4 + 32 * q4 + 4 * c) =
                  make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
        } else if (writers) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint4 w = make_uint4(pack2<T>(o[8 * c] * inv, o[8 * c + 1] * inv), pack2<T>(o[8 * c + 2] * inv, o[8 * c + 3] * inv),
                                 pack2<T>(o[8 * c + 4] * inv, o[8 * c + 5] * inv), pack2<T>(o[8 * c + 6] * inv, o[8 * c + 7] * inv));
            if (!some) w = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = w;
          }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int src = (lane >> 2) + 8 * j;
            const uint4 w = *reinterpret_cast<const uint4*>(stage + src * 64 + (((lane & 3) ^ ((src >> 1) & 3)) << 4));
            if ((writers >> src) & 1u)
              *reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + at_j[j] + 32 * q4 + 8 * (lane & 3)) = w;
          }
          __syncwarp();
        }
      }
      if (writer) {
        if (FORM == kGroups && !part) *reinterpret_cast<float2*>(whole) = make_float2(m_run, any ? s_run : 0.f);
        else if (!part && a.lse) a.lse[at / ZC_D] = some ? m_run + log2f(s_run) : -INFINITY;
        if (part)
          reinterpret_cast<float2*>(part + kItemRows * ZC_D * 4)[prow] = make_float2(m_run, any ? s_run : 0.f);
      }
      if (meet) {
        groups_sync();   // the second Q tile's place and the sums are free
        if (tid == 128) bar_arrive(&m_free[meetings & 1u]);
        ++meetings;
      }
      // this row's O is in registers or memory: the next item's products may overwrite it
      tc_fence_before();
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kCols) : "memory");
}

// Rows of the items that were worked on in pieces.  Block (c - 1) * 16 + i: rows 16 i ... of the item that the
// border before CTA c cuts first; a thread takes eight channels of a row.
template <typename T> __global__ void __launch_bounds__(256) k_chunk_join(const ChunkArgs k) {
  __shared__ int s_slot[ZC_PAGED_MAX_CTAS + 1], s_count;
  zc_let_next_start();
  zc_wait_for_last();
  const ZcPagedArgs& a = k.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const ChunkJoin j = k.ws.joins[blockIdx.x / 16 + 1];
  if (!j.on) return;
  // the pieces in order: the end of the share before the item's first border, then the starts behind each border;
  // as a rule there is one border
  if (warp == 0 && j.last > j.first) {
    int n = 1;
    if (lane == 0) s_slot[0] = 2 * (j.first - 1) + 1;
    for (int d = j.first; d <= j.last; d += 32) {
      const bool on = d + lane <= j.last && k.ws.used[d + lane];
      const unsigned m = __ballot_sync(0xffffffffu, on);
      if (on) s_slot[n + __popc(m & ((1u << lane) - 1u))] = 2 * (d + lane);
      n += __popc(m);
    }
    if (lane == 0) s_count = n;
  }
  if (j.last > j.first) __syncthreads();
  const int n = j.last > j.first ? s_count : 2;
  const int row = (int)(blockIdx.x % 16) * 16 + (threadIdx.x & 15), cg = threadIdx.x >> 4;
  const int g = row / kM, in = row % kM, tok_in = in / a.G, tok = j.tok0 + g * k.tpt + tok_in;
  if (tok_in >= k.tpt || tok >= j.n) return;
  auto piece = [&](int q) {
    return k.ws.parts + (long long)(j.last > j.first ? s_slot[q] : 2 * j.first - 1 + q) * kPartBytes;
  };
  auto sums = [&](int q) { return reinterpret_cast<const float2*>(piece(q) + kItemRows * ZC_D * 4)[row]; };
  struct Part { float4 x[2]; };
  auto channels = [&](int q) {
    const float4* p = reinterpret_cast<const float4*>(piece(q)) + row;
    Part r = {{p[cg * kItemRows], p[(cg + 16) * kItemRows]}};
    return r;
  };
  // the first two pieces (there always are) on their way together
  const float2 ms0 = sums(0), ms1 = sums(1);
  const Part p0 = channels(0), p1 = channels(1);
  float m = fmaxf(ms0.x, ms1.x);
#pragma unroll 4
  for (int q = 2; q < n; ++q) m = fmaxf(m, sums(q).x);
  float sum = 0.f;
  float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
  auto take = [&](float2 ms, const Part& p) {
    const float f = zc_exp2(ms.x - m);
    sum = fmaf(ms.y, f, sum);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      acc[u].x = fmaf(p.x[u].x, f, acc[u].x);
      acc[u].y = fmaf(p.x[u].y, f, acc[u].y);
      acc[u].z = fmaf(p.x[u].z, f, acc[u].z);
      acc[u].w = fmaf(p.x[u].w, f, acc[u].w);
    }
  };
  take(ms0, p0);
  take(ms1, p1);
#pragma unroll 2
  for (int q = 2; q < n; ++q) take(sums(q), channels(q));
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  const long long at = (long long)(j.row0 + tok) * a.h_q + j.kv * a.G + (in - tok_in * a.G);
#pragma unroll
  for (int u = 0; u < 2; ++u)
    *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.out) + at * ZC_D + 4 * (cg + 16 * u)) =
        make_uint2(pack2<T>(acc[u].x * inv, acc[u].y * inv), pack2<T>(acc[u].z * inv, acc[u].w * inv));
  if (a.lse && cg == 0) a.lse[at] = sum > 0.f ? m + log2f(sum) : -INFINITY;
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
// Places of the parts of a call's workspace; returns the bytes.
size_t carve(char* ws, ChunkWs* out) {
  size_t off = ZC_PAGES_SYNC_BYTES;   // the single-token kernel's counters stay as they are
  auto take = [&](size_t bytes) {
    char* p = ws + off;
    off += round_up(bytes);
    return p;
  };
  ChunkWs w;
  w.joins = (ChunkJoin*)take(ZC_PAGED_MAX_CTAS * sizeof(ChunkJoin));
  w.used = (int*)take(ZC_PAGED_MAX_CTAS * sizeof(int));
  w.parts = take((size_t)ZC_PAGED_MAX_CTAS * 2 * kPartBytes);
  if (out) *out = w;
  return off;
}

template <typename T, int FORM>
cudaError_t ready() {   // the shared memory the kernel asks for
  static std::atomic<unsigned long long> allowed{0};
  return zc_allow_smem(k_chunk_attention<T, FORM>, kSmem, &allowed);
}

// Dense K or V as pages: a batch row is a page of l tokens (64 channels, token, half of the channels, KV head,
// batch row), boxes of 64 tokens.
bool make_dense_map(CUtensorMap* map, const void* x, const zc_config& cfg, int l, const int64_t* ks) {
  const cuuint64_t dims[5] = {64, (cuuint64_t)l, 2, (cuuint64_t)cfg.n_kv_heads, (cuuint64_t)cfg.batch};
  const long long s[4] = {ks[2], 64, cfg.n_kv_heads > 1 ? ks[1] : ZC_D, cfg.batch > 1 ? ks[0] : ZC_D};
  cuuint64_t strides[4];
  for (int i = 0; i < 4; ++i) {
    if (s[i] <= 0 || (s[i] & 7)) return false;
    strides[i] = (cuuint64_t)s[i] * 2;
  }
  const cuuint32_t box[5] = {64, kN, 2, 1, 1};
  return zc_encode_map(map, cfg.dtype, 5, x, dims, strides, box);
}

template <typename T>
int launch_chunk(zc_pages* p, const ChunkArgs& k, const CUtensorMap& qmap, cudaStream_t st) {
  cudaError_t e = ready<T, kPages>();
  if (e != cudaSuccess) return e;
  e = zc_launch_early(k_chunk_attention<T, kPages>, dim3(p->n_sm), dim3(kThreads), kSmem, st, k, qmap, p->k64, p->v64);
  if (e != cudaSuccess) return e;
  p->launches += 1;
  if (p->n_sm > 1) {
    e = zc_launch_early(k_chunk_join<T>, dim3(16 * (p->n_sm - 1)), dim3(256), 0, st, k);
    if (e != cudaSuccess) return e;
    p->launches += 1;
  }
  return cudaSuccess;
}

template <typename T>
cudaError_t launch_groups(zc_pages* p, const ChunkArgs& k, const CUtensorMap& qmap, cudaStream_t st) {
  const cudaError_t e = ready<T, kGroups>();
  if (e != cudaSuccess) return e;
  return zc_launch_early(k_chunk_attention<T, kGroups>, dim3(p->n_sm), dim3(kThreads), kSmem, st, k, qmap, p->k64, p->v64);
}

// Items that a head can have: whole ones, and a part of one for each group.
int most_items(int G, int n_groups, int n_rows) { return n_rows / (2 * tokens_per_tile(G)) + n_groups; }

// Places of the parts of a shared call's workspace, behind a chunk call's; returns the bytes.
size_t carve_groups(const zc_page_config& c, int n_req, int n_rows, char* ws, ZcGroups* gr) {
  const int G = c.n_q_heads / c.n_kv_heads;
  size_t off = carve(nullptr, nullptr);
  auto take = [&](size_t bytes) {
    char* p = ws + off;
    off += round_up(bytes);
    return p;
  };
  ZcGroups g;
  memset(&g, 0, sizeof(g));
  g.told = (int*)ws + ZC_PAGED_MAX_CTAS + 2;
  g.head = (int*)take(sizeof(int));
  g.keys = (int*)take(kMaxGroups * sizeof(int));
  g.lead = (int*)take(kMaxGroups * sizeof(int));
  g.last = (int*)take(ZC_PAGED_MAX_CTAS * sizeof(int));
  g.info = (int4*)take((size_t)n_req * sizeof(int4));
  g.own = (int4*)take((size_t)n_req * sizeof(int4));
  g.cut = (int*)take((size_t)most_items(G, n_req, n_rows) * c.n_kv_heads * sizeof(int));
  const size_t row = (size_t)c.n_q_heads * ZC_PART_STRIDE * 4;
  g.rows = (float*)take(n_rows * row);
  g.own_line = (long long*)take(2 * sizeof(long long));
  // (a request's rows, and as many again for each warp, where the next one goes on)
  g.own_rows = (float*)take(n_rows * row + (size_t)kOwnWarps * ZC_PAGED_MAX_CTAS * ZC_PAGED_ROWS * ZC_PART_STRIDE * 4);
  if (gr) *gr = g;
  return off;
}

}  // namespace

size_t zc_paged_shared_workspace(const zc_page_config& c, int n_req, int n_rows) {
  return carve_groups(c, n_req, n_rows, nullptr, nullptr);
}

int zc_launch_paged_shared(zc_pages* p, const ZcPagedArgs& a, const int32_t* group_start, const int32_t* shared_len,
                           int n_groups, float* logits, char* ws, cudaStream_t st) {
  if (!zc_page_maps(p)) return (int)cudaErrorNotSupported;
  ChunkArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  carve(ws, &k.ws);
  carve_groups(p->cfg, a.n_req, a.n_rows, ws, &k.gr);
  k.gr.start = group_start;
  k.gr.shared = shared_len;
  k.gr.n = n_groups;
  k.gr.most = most_items(a.G, n_groups < a.n_req ? n_groups : a.n_req, a.n_rows);
  k.gr.used = k.ws.used;
  k.gr.parts = k.ws.parts;
  k.tpt = tokens_per_tile(a.G);
  k.o_row = (long long)a.h_q * ZC_D;
  k.o_head = ZC_D;
  CUtensorMap qmap;
  memset(&qmap, 0, sizeof(qmap));
  if (!make_q_map(&qmap, a.q, p->cfg.dtype, a.h_q, a.G, a.n_rows, 1, a.qs_head, a.qs_row, 0))
    return (int)cudaErrorNotSupported;
  // The first kernel sets gr.told, the joining one clears it: what can fail without a launch does so before the first, and
  // where a launch behind it fails, the word is cleared all the same (left set, it would mislead the next call's kernels).
  int e = zc_launch_own_keys(p, a, k.gr, k.tpt, logits, false, st);
  if (e != cudaSuccess) return e;
  e = p->cfg.dtype == ZC_F16 ? launch_groups<__half>(p, k, qmap, st) : launch_groups<__nv_bfloat16>(p, k, qmap, st);
  if (e != cudaSuccess) return e;
  p->launches += 1;
  e = zc_launch_own_keys(p, a, k.gr, k.tpt, logits, true, st);
  if (e != cudaSuccess) cudaMemsetAsync(k.gr.told, 0, sizeof(int), st);
  return e;
}

size_t zc_paged_chunk_workspace() { return carve(nullptr, nullptr); }

bool zc_paged_chunk_fits(int G, int n_req, int n_rows) {
  return (long long)n_rows / (2 * tokens_per_tile(G)) + n_req <= kMaxItems;
}

int zc_launch_paged_chunk(zc_pages* p, const ZcPagedArgs& a, char* ws, cudaStream_t st) {
  if (!zc_page_maps(p)) return (int)cudaErrorNotSupported;
  ChunkArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  carve(ws, &k.ws);
  k.tpt = tokens_per_tile(a.G);
  k.o_row = (long long)a.h_q * ZC_D;
  k.o_head = ZC_D;
  CUtensorMap qmap;
  memset(&qmap, 0, sizeof(qmap));
  if (!make_q_map(&qmap, a.q, p->cfg.dtype, a.h_q, a.G, a.n_rows, 1, a.qs_head, a.qs_row, 0))
    return (int)cudaErrorNotSupported;
  return p->cfg.dtype == ZC_F16 ? launch_chunk<__half>(p, k, qmap, st) : launch_chunk<__nv_bfloat16>(p, k, qmap, st);
}

int zc_launch_prefill_window(zc_cache* c, const void* Q, const void* K, const void* V, int l, const int64_t* qs,
                             const int64_t* ks, int window, int sinks, void* O, float* lse, cudaStream_t st) {
  const zc_config& cfg = c->cfg;
  ChunkArgs k;
  memset(&k, 0, sizeof(k));
  k.a.n_req = cfg.batch;
  k.a.h_q = cfg.n_q_heads;
  k.a.h_kv = cfg.n_kv_heads;
  k.a.G = c->lay.G;
  k.a.window = window;
  k.a.sinks = sinks;
  k.a.out = O;
  k.a.lse = lse;
  k.tpt = tokens_per_tile(k.a.G);
  k.l = l;
  k.items = zc_ceil_div(l, 2 * k.tpt);
  k.o_row = ZC_D;
  k.o_head = (long long)l * ZC_D;
  k.o_req = (long long)cfg.n_q_heads * l * ZC_D;
  CUtensorMap qmap, kmap, vmap;
  memset(&qmap, 0, sizeof(qmap));
  memset(&kmap, 0, sizeof(kmap));
  memset(&vmap, 0, sizeof(vmap));
  if (!make_q_map(&qmap, Q, cfg.dtype, cfg.n_q_heads, k.a.G, l, cfg.batch, qs[1], qs[2], qs[0]) ||
      !make_dense_map(&kmap, K, cfg, l, ks) || !make_dense_map(&vmap, V, cfg, l, ks))
    return (int)cudaErrorNotSupported;
  const long long n = (long long)k.items * cfg.batch * cfg.n_kv_heads;
  const int grid = n < c->n_sm ? (int)n : c->n_sm;
  cudaError_t e;
  if (cfg.dtype == ZC_F16) {
    e = ready<__half, kDense>();
    if (e != cudaSuccess) return e;
    e = zc_launch_early(k_chunk_attention<__half, kDense>, dim3(grid), dim3(kThreads), kSmem, st, k, qmap, kmap, vmap);
  } else {
    e = ready<__nv_bfloat16, kDense>();
    if (e != cudaSuccess) return e;
    e = zc_launch_early(k_chunk_attention<__nv_bfloat16, kDense>, dim3(grid), dim3(kThreads), kSmem, st, k, qmap, kmap, vmap);
  }
  c->launches += 1;
  return (int)e;
}

int zc_paged_chunk_error_code(int* out) { return (int)cudaMemcpyFromSymbol(out, g_zc_tc_error, sizeof(int)); }
