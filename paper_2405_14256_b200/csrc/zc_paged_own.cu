// Attention of requests that begin alike (few rows each): their own keys, behind those that their group shares, and the
// joining of the two.
//
// k_own_keys runs beside the kernel of the shared keys, on the SMs that that one leaves (zc_paged_groups.cuh).  Own parts
// are short as a rule, so a piece of some blocks of 16 keys is one warp's alone: no warp waits for another, and
// nothing is joined inside a CTA (eight warps to a unit, whose results meet in shared memory: 5 us of a CTA per (request, KV
// head) of some 300 keys).  The blocks of all KV heads and requests lie on one line, each (KV head, request) with what a
// piece costs beside its blocks, and every warp has an equal stretch of it: the end of one request's, whole ones, the
// beginning of another's (pieces of one length dealt out to the warps in turn left half of them idle at the end: 108 us for
// 128 requests of up to 2048 own keys behind 30000, 95 so).  A warp works out 32 of its pieces at a time, a lane each, and
// runs through their blocks with a ring of three stages (16 keys and 16 values each, bulk tensor copies), ahead of itself
// across pieces.  Every piece leaves (maximum, sum, 128 sums) per row.
// k_own_join puts a row's pieces and its group's together, in their order.  Bound: HBM, every own key and value once.
#include <cstring>
#include "zc_paged_block.cuh"
#include "zc_paged_groups.cuh"

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
static_assert(kOwnWarps == 2 * kWarps, "two CTAs to an SM");
constexpr int kStages = 3;
constexpr int kRing = kWarps * kStages * 2 * kHalf;    // 96 KB: two CTAs to an SM
constexpr int kBatch = 32;                             // pieces that a warp knows
constexpr int kPieceCost = 4;                          // what a piece costs beside its blocks, in blocks
constexpr int kLeastStretch = 4 + kPieceCost;          // of a warp, in blocks
constexpr int kStride = ZC_PART_STRIDE;

struct Piece {
  int r, kv, row0, n, p0;     // request (-1: no more), KV head, its rows, the position of the first
  int key0, key1;             // keys: whole blocks, the last one's end may lie behind the request's
  int lo, base;               // first own key of the request; where the piece's rows are among all pieces' rows
};
constexpr int kPieceInts = 9;   // (odd: lanes write without conflicts)
static_assert(sizeof(Piece) == kPieceInts * 4, "a piece");
constexpr int kSmem = kRing + kWarps * kStages * 8 + kWarps * kBatch * kPieceInts * 4 + 64 + 1024;   // 1 KB: alignment
static_assert(GroupTables::kInts * 4 <= kRing, "the groups' tables, before the first copy");
// Of each request (kPlanReq of them at most; else in global memory): where its blocks begin on a KV head's line (64 bits),
// its group's keys.
constexpr int kOwnSmem = kSmem + 3 * kPlanReq * 4;

struct OwnArgs {
  ZcPagedArgs a;
  ZcGroups gr;
  int tpt, n_sm;
  float* logits;
};

__device__ __forceinline__ int own_keys(const Chunk& c, int shared) { return max(0, c.p0 + c.n - shared); }
// A request's length on the line, in blocks; the piece that it has in any case, of no key maybe, costs as well.
__device__ __forceinline__ int own_length(const Chunk& c, int shared) {
  return c.n > 0 ? (int)(((long long)own_keys(c, shared) + kBlk - 1) / kBlk) + kPieceCost : 0;
}

// Where each request's blocks begin on a KV head's line, for every CTA by itself (left in global memory, by every CTA the
// same, where it reads them again).  Returns the line's length.
__device__ __forceinline__ long long plan_line(const OwnArgs& k, const GroupTables& t, long long* s_warp, long long* s_at,
                                               int* s_shared) {
  const ZcPagedArgs& a = k.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  long long line = 0;
  for (int c0 = 0; c0 < a.n_req; c0 += kThreads) {
    const int r = c0 + tid;
    int length = 0, shared = 0;
    if (r < a.n_req) {
      shared = t.keys_of(r);
      length = own_length(t.chunk(a, r), shared);
    }
    long long x = length;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += u;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    long long before = line + x - length;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += s_warp[w];
      line += s_warp[w];
    }
    if (r < a.n_req) {
      if (t.held) {
        s_at[r] = before;
        s_shared[r] = shared;
      }
      if (!t.held || blockIdx.x == 0) k.gr.own[r] = make_int4((int)before, (int)(before >> 32), shared, length);
    }
  }
  __syncthreads();   // (a thread reads what others of its CTA have written)
  return line;
}
__device__ __forceinline__ long long line_at(const int4& own) { return (long long)own.y << 32 | (uint32_t)own.x; }

template <typename T, int NT, bool WEIGHTS>
__global__ void __launch_bounds__(kThreads, 2)
    k_own_keys(const OwnArgs k, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  const ZcPagedArgs& a = k.a;
  const uint32_t raw_u = zc_smem_u32(smem_raw);
  const uint32_t base_u = (raw_u + 1023u) & ~1023u;
  char* base = smem_raw + (base_u - raw_u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + kRing);
  int* s_pieces = reinterpret_cast<int*>(bars + kWarps * kStages);
  long long* s_warp = reinterpret_cast<long long*>(s_pieces + kWarps * kBatch * kPieceInts);
  long long* s_at = s_warp + 8;
  int* s_shared = reinterpret_cast<int*>(s_at + kPlanReq);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < kWarps * kStages) bar_init(&bars[tid], 1);
  if (tid == 64) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&kmap)));
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&vmap)));
  }
  asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  zc_let_next_start();
  // This kernel does not wait for the one of the shared keys, whose CTAs started once all before them was complete; it takes
  // the SMs that that one leaves.  Its first CTA waits at its end, so that what comes behind waits for both.
  // (CTAs that find no SM before others leave theirs are not needed as a rule, and need not work that out)
  const int told = *reinterpret_cast<volatile int*>(k.gr.told);
  if (told > 0 && blockIdx.x > 0 && (int)blockIdx.x >= 2 * (k.n_sm - (told - 1))) return;
  const GroupTables tables(base, k.gr.n, a.n_req);
  const int sms = k.n_sm - plan_groups<kThreads>(a, k.gr, tables, k.tpt, k.n_sm);
  const int n_warps = sms * kOwnWarps, wid = blockIdx.x * kWarps + warp;
  const long long line = plan_line(k, tables, s_warp, s_at, s_shared), total = line * a.h_kv;
  const long long stretch = max((long long)kLeastStretch, (total + n_warps - 1) / n_warps);
  if (blockIdx.x == 0 && tid == 0) {
    k.gr.own_line[0] = line;
    k.gr.own_line[1] = stretch;
  }
  const bool held = tables.held;
  async_proxy_fence();   // the tables' place is the ring's from here on, whose copies come by the other proxy
  __syncthreads();

  if (wid < n_warps) {
    // ---- pieces: 32 at a time, a lane each ----
    int* mine = s_pieces + warp * kBatch * kPieceInts;
    long long x0 = min(total, wid * stretch);
    const long long x1 = min(total, x0 + stretch);
    auto find = [&]() {   // those from x0 on
      const int kv0 = (int)(x0 / line);
      const long long rem = x0 - kv0 * line;
      int lo = 0, hi = a.n_req;   // the last request that begins at or before this place
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if ((held ? s_at[m] : line_at(k.gr.own[m])) <= rem) lo = m; else hi = m;
      }
      const int unit = kv0 * a.n_req + lo + lane;
      Piece p;
      p.r = -1;
      p.kv = unit / a.n_req;
      const int r = unit - p.kv * a.n_req;
      long long end = 0;
      if (p.kv < a.h_kv) {
        const Chunk c = load_chunk(a, r);
        const int4 own = held ? make_int4(0, 0, s_shared[r], 0) : k.gr.own[r];
        const long long at = p.kv * line + (held ? s_at[r] : line_at(own)), from = max(at, x0);
        end = min(at + own_length(c, own.z), x1);
        if (from < end) {
          p.r = r;
          p.row0 = c.row0;
          p.n = c.n;
          p.p0 = c.p0;
          p.lo = own.z;
          p.key0 = own.z + kBlk * max(0, (int)(from - at) - kPieceCost);
          p.key1 = (int)min((long long)own.z + kBlk * (long long)max(0, (int)(end - at) - kPieceCost),
                            (long long)own.z + own_keys(c, own.z));
          // (each next piece is the next warp's or of the next rows: no two have the same place)
          p.base = (p.kv * a.n_rows + c.row0) * a.G + wid * ZC_PAGED_ROWS;
        }
      }
      const unsigned on = __ballot_sync(0xffffffffu, p.r >= 0);
      __syncwarp();
      if (lane >= __popc(on)) mine[lane * kPieceInts] = -1;
      if (p.r >= 0) {
        int* to = mine + __popc(on & ((1u << lane) - 1u)) * kPieceInts;
        const int* src = reinterpret_cast<const int*>(&p);
#pragma unroll
        for (int e = 0; e < kPieceInts; ++e) to[e] = src[e];
      }
      x0 = on ? __shfl_sync(0xffffffffu, end, 31 - __clz(on)) : x1;
      __syncwarp();
    };
    auto piece = [&](int i) {
      Piece p;
      int* to = reinterpret_cast<int*>(&p);
      const int* src = mine + i * kPieceInts;
#pragma unroll
      for (int e = 0; e < kPieceInts; ++e) to[e] = src[e];
      return p;
    };
    const uint32_t ring = base_u + warp * kStages * 2 * kHalf;
    uint64_t* full = bars + warp * kStages;
    bool ok = true;      // no wait of the warp has run out
    int stage = 0;
    uint32_t phase = 0;
    const int quad = lane & 3, oct = lane >> 2;
    while (x0 < x1) {
      find();
      // ---- copies, running ahead of the warp's own blocks within these pieces ----
      int pi = 0, pkey = 0, at_key = -1, at_kv = 0, page = 0;   // the next block: its page id is asked for now and used then
      Piece pp = piece(0);
      pkey = pp.key0;
      auto fetch = [&]() {
        for (;;) {
          if (pi == kBatch || pp.r < 0) {
            at_key = -1;
            return;
          }
          if (pkey < pp.key1) {
            at_key = pkey;
            at_kv = pp.kv;
            page = a.table[(long long)pp.r * a.table_width + (pkey >> a.page_log2)];
            pkey += kBlk;
            return;
          }
          if (++pi < kBatch) {
            pp = piece(pi);
            pkey = pp.key0;
          }
        }
      };
      int held[kStages];   // pages of the blocks in the stages
#pragma unroll
      for (int i = 0; i < kStages; ++i) held[i] = -1;
      auto issue = [&](int s) {
        if (at_key < 0) return;
#pragma unroll
        for (int i = 0; i < kStages; ++i)
          if (WEIGHTS && i == s) held[i] = page;
        if (lane == 0) {
          const int id = page >= 0 && page < a.n_pages ? page : a.n_pages;   // beyond the pool: arrives as zeros
          const int row = at_key & ((1 << a.page_log2) - 1);
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(zc_smem_u32(&full[s])),
                       "r"(2 * kHalf)
                       : "memory");
          const uint32_t dst = ring + s * 2 * kHalf;
          page_copy(&kmap, dst, &full[s], row, 0, at_kv, id);
          page_copy(&vmap, dst + kHalf, &full[s], row, 0, at_kv, id);
        }
        fetch();
      };
      fetch();
#pragma unroll
      for (int i = 0; i < kStages; ++i)
        if (ok) issue((stage + i) % kStages);
      // ---- the pieces, their query rows asked for one ahead ----
      Piece p = piece(0);
      uint32_t qf[NT][8][2], qn[NT][8][2];
      load_rows<T, NT>(a, p.row0, p.kv, p.n * a.G, qn);
#pragma unroll 1
      for (int i = 0; i < kBatch && p.r >= 0; ++i) {
        const Piece now = p;
        const int rows = now.n * a.G, p_last = now.p0 + now.n - 1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            qf[nt][ks][0] = qn[nt][ks][0];
            qf[nt][ks][1] = qn[nt][ks][1];
          }
        if (i + 1 < kBatch) p = piece(i + 1);
        if (i + 1 < kBatch && p.r >= 0) load_rows<T, NT>(a, p.row0, p.kv, p.n * a.G, qn);
        int pos[NT][2];
        row_positions<NT>(a, now.p0, rows, pos);
        ZcSeen seen;
        seen.lo = now.lo;
        seen.hi = p_last + 1;
        seen.sink_n = seen.nsb = seen.wb0 = seen.nb = 0;
        RowState<NT> x;
        x.clear();
#pragma unroll 1
        for (int key0 = now.key0; ok && key0 < now.key1; key0 += kBlk) {
          ok = warp_wait(&full[stage], phase);
          if (!ok) break;   // nothing more is copied
          const uint32_t kt = ring + stage * 2 * kHalf, vt = kt + kHalf;
          float* keep = nullptr;
          if (WEIGHTS) {
            int id = -1;
#pragma unroll
            for (int s = 0; s < kStages; ++s)
              if (s == stage) id = held[s];
            if (id >= 0 && id < a.n_pages) keep = logits_of(k.logits, a, id, now.kv, key0);
          }
          attend_block<T, NT, WEIGHTS>(x, qf, pos, kt, vt, base + (vt - base_u), key0, now.p0, p_last, seen, a, rows, keep);
          __syncwarp();
          issue(stage);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        // ---- what the piece's rows have ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float sum = x.s[nt][e];
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
            const int row = 8 * nt + 2 * quad + e;
            if (row >= rows) continue;
            float* to = k.gr.own_rows + (long long)(now.base + row) * kStride;
            if (oct == 0) *reinterpret_cast<float2*>(to) = make_float2(x.m[nt][e], sum);
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) {
              to[4 + 16 * mt + oct] = x.o[nt][mt][e];
              to[4 + 16 * mt + oct + 8] = x.o[nt][mt][e + 2];
            }
          }
      }
    }
    if (!ok)   // the copies that were on their way
      for (int i = 0; i < kStages; ++i) drain(&full[i], i < stage ? phase ^ 1u : phase);
  }
  if (blockIdx.x == 0) zc_wait_for_last();
}

// A row's pieces of its own keys, and of its group's, to its output.  A warp has ROWS consecutive rows (token * G + head) of
// a request and KV head, 32 / ROWS lanes to a row, a lane one or two groups of four channels (with eight or four rows the
// channels are four or two warps'), and four pieces on their way at a time.  A warp to all channels of a row, piece by
// piece, or of eight rows, took 17 to 19 us of 64 rows and 32 heads; eight rows to a warp with one row to a unit 25 us of 131
// rows and 32 heads.
struct JoinArgs {
  ZcPagedArgs a;
  ZcGroups gr;
  int tpt, per_unit;                // per_unit: warps to a (request, KV head)
};
template <typename T, int ROWS> __global__ void __launch_bounds__(256) k_own_join(const JoinArgs k) {
  constexpr int kLanes = 32 / ROWS, kVec = ROWS == 1 ? 1 : 2, kParts = 32 / (kLanes * kVec);   // groups of channels: 32
  zc_let_next_start();
  const ZcPagedArgs& a = k.a;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int blk = (int)(w % k.per_unit), unit = (int)(w / k.per_unit);
  const int r = unit / a.h_kv, kv = unit - r * a.h_kv;
  Chunk c;
  c.row0 = c.n = c.p0 = 0;
  if (r < a.n_req) c = load_chunk(a, r);   // (what came before the two kernels is complete)
  zc_wait_for_last();
  if (blockIdx.x == 0 && threadIdx.x == 0) *k.gr.told = 0;   // as the next call wants it
  if (c.n <= 0) return;
  const int4 own = k.gr.own[r], info = k.gr.info[r];
  const int row = blk / kParts * ROWS + lane % ROWS;
  const int cg = blk % kParts * (kLanes * kVec) + lane / ROWS;   // this lane's groups of channels: cg, cg + kLanes
  const int t = row / a.G, head = kv * a.G + row - t * a.G;
  if (t >= c.n) return;
  // its pieces: the warps that have a part of its stretch of the line
  const long long at0 = kv * k.gr.own_line[0] + line_at(own), stretch = k.gr.own_line[1];
  const int w0 = (int)(at0 / stretch), n_own = (int)((at0 + own.w - 1) / stretch) - w0 + 1;
  float m = kNoMax, sum = 0.f;
  float4 acc[kVec];
#pragma unroll
  for (int j = 0; j < kVec; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  auto take = [&](float2 ms, const float4 (&x)[kVec]) {
    const float top = fmaxf(m, ms.x), fo = zc_exp2(m - top), fn = zc_exp2(ms.x - top);
    m = top;
    sum = fmaf(sum, fo, ms.y * fn);
#pragma unroll
    for (int j = 0; j < kVec; ++j)
      acc[j] = make_float4(fmaf(acc[j].x, fo, x[j].x * fn), fmaf(acc[j].y, fo, x[j].y * fn), fmaf(acc[j].z, fo, x[j].z * fn),
                           fmaf(acc[j].w, fo, x[j].w * fn));
  };
  // the group's keys: where their result is
  const int n_cta = *k.gr.head;
  const int tok = info.y + t, tpi = 2 * k.tpt, in_group = tok / tpi, tok_in = tok - in_group * tpi;
  const int item = info.z + in_group, half = tok_in >= k.tpt;
  const int prow = half * kM + (tok_in - half * k.tpt) * a.G + head - kv * a.G;
  const bool shared = info.x > 0 && item < k.gr.most;   // (beyond: lengths that contradict one another)
  const int cut = shared ? k.gr.cut[(long long)item * a.h_kv + kv] : 0;
  const bool pieces = shared && cut > 0 && cut < n_cta;
  const int last = pieces ? min(k.gr.last[cut], n_cta - 1) : 0;
  // own keys, four pieces at a time
  const float* from = k.gr.own_rows + ((long long)(kv * a.n_rows + c.row0) * a.G + w0 * ZC_PAGED_ROWS + row) * kStride;
  constexpr int next = ZC_PAGED_ROWS * kStride;
  for (int p0 = 0; p0 < n_own; p0 += 4) {
    float2 ms[4];
    float4 x[4][kVec];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (p0 + u < n_own) {
        const float* at = from + (p0 + u) * next;
        ms[u] = *reinterpret_cast<const float2*>(at);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[u][j] = *reinterpret_cast<const float4*>(at + 4 + 4 * (cg + kLanes * j));
      }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (p0 + u < n_own) take(ms[u], x[u]);
  }
  if (pieces) {
    // in order: the end of the share before the item's first border, then the starts behind each border
    for (int d0 = cut - 1; d0 <= last; d0 += 4) {
      float2 ms[4];
      float4 x[4][kVec];
      bool on[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (d0 + u <= last) {
          const int d = d0 + u;
          const char* at = k.gr.parts + (long long)(d < cut ? 2 * d + 1 : 2 * d) * ZC_CHUNK_PART_BYTES;
          on[u] = d < cut || k.gr.used[d];
          ms[u] = reinterpret_cast<const float2*>(at + ZC_CHUNK_PART_ROWS * ZC_D * 4)[prow];
#pragma unroll
          for (int j = 0; j < kVec; ++j)
            x[u][j] = reinterpret_cast<const float4*>(at)[(cg + kLanes * j) * ZC_CHUNK_PART_ROWS + prow];
        }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (d0 + u <= last && on[u]) take(ms[u], x[u]);
    }
  } else if (shared) {
    const float* at = k.gr.rows + ((long long)(c.row0 + t) * a.h_q + head) * kStride;
    float4 x[kVec];
    const float2 ms = *reinterpret_cast<const float2*>(at);
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[j] = *reinterpret_cast<const float4*>(at + 4 + 4 * (cg + kLanes * j));
    take(ms, x);
  }
  const long long at = (long long)(c.row0 + t) * a.h_q + head;
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int j = 0; j < kVec; ++j)
    *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.out) + at * ZC_D + 4 * (cg + kLanes * j)) =
        make_uint2(pack2<T>(acc[j].x * inv, acc[j].y * inv), pack2<T>(acc[j].z * inv, acc[j].w * inv));
  if (a.lse && cg == 0) a.lse[at] = sum > 0.f ? m + log2f(sum) : -INFINITY;
}

template <typename T, int ROWS> cudaError_t launch_join(const JoinArgs& j, cudaStream_t st) {
  JoinArgs k = j;
  constexpr int kParts = ROWS == 8 ? 4 : ROWS == 4 ? 2 : 1;
  k.per_unit = (j.a.max_rows * j.a.G + ROWS - 1) / ROWS * kParts;
  const long long blocks = ((long long)k.a.n_req * k.a.h_kv * k.per_unit + 7) / 8;
  return zc_launch_early(k_own_join<T, ROWS>, dim3((unsigned)blocks), dim3(256), 0, st, k);
}
template <typename T> cudaError_t launch_join_rows(const JoinArgs& j, cudaStream_t st) {
  const int rows = j.a.max_rows * j.a.G;
  return rows > 4 ? launch_join<T, 8>(j, st) : rows > 2 ? launch_join<T, 4>(j, st) : rows > 1 ? launch_join<T, 2>(j, st)
                                                                                              : launch_join<T, 1>(j, st);
}

template <typename T, int NT, bool WEIGHTS>
cudaError_t launch(zc_pages* p, const OwnArgs& k, bool go, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = zc_allow_smem(k_own_keys<T, NT, WEIGHTS>, kOwnSmem, &allowed);
  if (e != cudaSuccess || !go) return e;
  return zc_launch_early(k_own_keys<T, NT, WEIGHTS>, dim3(2 * k.n_sm), dim3(kThreads), kOwnSmem, st, k, p->k16, p->v16);
}
template <typename T, int NT> cudaError_t launch_mode(zc_pages* p, const OwnArgs& k, bool go, cudaStream_t st) {
  return k.logits ? launch<T, NT, true>(p, k, go, st) : launch<T, NT, false>(p, k, go, st);
}
template <typename T> cudaError_t launch_rows(zc_pages* p, const OwnArgs& k, bool go, cudaStream_t st) {
  return k.a.max_rows * k.a.G <= 8 ? launch_mode<T, 1>(p, k, go, st) : launch_mode<T, 2>(p, k, go, st);
}

}  // namespace

int zc_launch_own_keys(zc_pages* p, const ZcPagedArgs& a, const ZcGroups& gr, int tpt, float* logits, bool go,
                       cudaStream_t st) {
  OwnArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  k.gr = gr;
  k.tpt = tpt;
  k.n_sm = p->n_sm;
  k.logits = logits;
  const bool half = p->cfg.dtype == ZC_F16;
  cudaError_t e = half ? launch_rows<__half>(p, k, go, st) : launch_rows<__nv_bfloat16>(p, k, go, st);
  if (e != cudaSuccess || !go) return (int)e;
  p->launches += 1;
  JoinArgs j;
  memset(&j, 0, sizeof(j));
  j.a = a;
  j.gr = gr;
  j.tpt = tpt;
  e = half ? launch_join_rows<__half>(j, st) : launch_join_rows<__nv_bfloat16>(j, st);
  if (e == cudaSuccess) p->launches += 1;
  return (int)e;
}

int zc_paged_own_error_code(int* out) { return (int)cudaMemcpyFromSymbol(out, g_zc_tc_error, sizeof(int)); }
