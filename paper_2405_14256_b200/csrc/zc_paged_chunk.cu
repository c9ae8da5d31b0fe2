// Attention of chunks of new tokens over pages, and of whole prompts in dense tensors under a sliding
// window (Eq. 2 with its causal mask; bound: tensor cores, and one exp2 per visible pair).
//
// The query heads of a KV head are packed beside each other: row = token * G + head, 128 / G tokens to
// a tile of 128 rows, so that short chunks fill the tile, a key tile is read once for the whole group and
// little work falls on tiles that the causal mask or the window cuts.  A work item is two such tiles
// (groups 0 and 1) of one request and KV head, and the key tiles (128 keys) that any of its rows sees:
// those of the first `sinks` tokens, then those of the window.  Items go through the kernel of
// persistent CTAs one after the other:
//   warp 0   the matrix products, tcgen05.mma with accumulators in tensor memory:
//            S_g = Q_g K^T (both K-major in shared memory), O_g += P_g V (P_g in tensor memory over
//            the first 64 columns of S_g, V with its channels contiguous)
//   warp 1   the copies: Q by one box per tile half, K and V page by page (a lane per page)
//   warps 4-7, 8-11  groups 0 and 1, one row per thread: running maximum (O rescaled when it grows by
//            more than 8, base 2) and sum in fp32, P rounded to the input type, output and log-sum-exp
// While one group turns S into P the tensor cores work for the other; the next item's Q and first key
// tiles arrive while this one's output is written.
// For pages the list of items is made on the device (k_chunk_plan: lengths stay there).  Where a call has
// few items for the GPU, those with many key tiles are cut into pieces along the keys, and k_chunk_join
// puts the pieces together in their order.
#include <cstring>
#include "zc_paged.cuh"
#include "zc_layout.cuh"

namespace {

constexpr int kThreads = 384;
constexpr int kKS = 3, kVS = 2;                       // key and value buffers
constexpr uint32_t kCols = 512;                       // S_0 | S_1 | O_0 | O_1
constexpr int kTiles = (2 + kKS + kVS) * kTile;       // 224 KB
constexpr int kSmem = kTiles + 1024 + 256;
constexpr float kTau = 8.f;
constexpr float kNoMax = -1e30f;
constexpr int kTileLog2 = 7;
constexpr int kPartStride = ZC_PART_STRIDE;           // m, sum, -, -, acc[128]
constexpr int kItemRows = 2 * kM;
// Pieces: at most kPieces key-tile ranges of full length over all heads, and no more remainders.
constexpr int kPieces = 2 * ZC_PAGED_MAX_CTAS;
constexpr int kMaxSlots = 2 * kPieces;
constexpr int kPlanThreads = 1024;

// One piece of work: tokens tok0 ... of request r (one item), key tiles t0 .. t1 - 1 of those it sees.
struct ChunkWork {
  int r, tok0, t0, t1;
  int slot;        // -1: the whole item; else its partial results' place among one head's
  int pad[3];
};
struct ChunkJoin { int r, tok0, slot, n; };
struct ChunkHead { int n_work, n_join, slots_per_head, pad; };

struct ChunkWs {
  ChunkHead* head;
  int* item_start;    // [n_req + 1] items before a request
  ChunkWork* work;
  ChunkJoin* joins;
  float* parts;       // [slot][256][132]
};

struct ChunkArgs {
  ZcPagedArgs a;
  ChunkWs ws;
  long long o_req, o_row, o_head;      // elements: out; the log-sum-exp's are these / 128
  int tpt;                             // tokens per tile
  int l, items;                        // dense form: tokens per batch row, items per (batch row, KV head)
};

// A request's chunk as the kernels see it.
struct Chunk { int row0, n, p0; };
__device__ __forceinline__ Chunk load_chunk(const ZcPagedArgs& a, int r) {
  const int e0 = min(max(a.row_start[r], 0), a.n_rows);
  const int e1 = min(max(a.row_start[r + 1], e0), a.n_rows);
  const long long cap = (long long)a.table_width << a.page_log2;
  const int kv = (int)min((long long)max(a.kv_len[r], 0), cap);
  Chunk c;
  c.row0 = e0;
  c.n = min(e1 - e0, a.max_rows);
  c.p0 = kv - (e1 - e0);
  return c;
}
__device__ __forceinline__ int item_tiles(const ZcPagedArgs& a, const Chunk& c, int tok0, int tpi) {
  const int last = min(tok0 + tpi, c.n) - 1;
  return zc_seen(c.p0 + tok0, c.p0 + last, a.window, a.sinks, kTileLog2).nb;
}

__device__ __forceinline__ int block_scan(int v, int* s_warp, int* total) {   // exclusive, kPlanThreads threads
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
  if (warp == 0) {
    int w = s_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  *total = s_warp[31];
  return incl - v + (warp ? s_warp[warp - 1] : 0);
}

// The list of work of one KV head (every head has the same), and the items that are in pieces.
// One CTA; lengths are read here and nowhere on the host.
__global__ void __launch_bounds__(kPlanThreads, 1) k_chunk_plan(const ChunkArgs k, int n_cta) {
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  __shared__ int s_warp[32];
  __shared__ long long s_tiles;
  const ZcPagedArgs& a = k.a;
  const int tid = threadIdx.x, tpi = 2 * k.tpt;
  if (tid == 0) s_tiles = 0;
  int items = 0;
  for (int c0 = 0; c0 < a.n_req; c0 += kPlanThreads) {
    int n = 0;
    if (c0 + tid < a.n_req) n = (load_chunk(a, c0 + tid).n + tpi - 1) / tpi;
    int t;
    const int at = block_scan(n, s_warp, &t);
    if (c0 + tid < a.n_req) k.ws.item_start[c0 + tid] = items + at;
    items += t;
  }
  if (tid == 0) k.ws.item_start[a.n_req] = items;
  __syncthreads();
  auto find = [&](int i, int* tok0) {   // request and first token of item i
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (k.ws.item_start[m] <= i) lo = m; else hi = m;
    }
    *tok0 = (i - k.ws.item_start[lo]) * tpi;
    return lo;
  };
  long long tiles = 0;
  for (int i = tid; i < items; i += kPlanThreads) {
    int tok0;
    const int r = find(i, &tok0);
    tiles += item_tiles(a, load_chunk(a, r), tok0, tpi);
  }
  atomicAdd(reinterpret_cast<unsigned long long*>(&s_tiles), (unsigned long long)tiles);
  __syncthreads();
  // Pieces: where the items of all heads come to fewer than four per CTA, none is longer than half a
  // CTA's even share (so that the busiest CTA ends within about half a share of the others), and no
  // shorter than 4 tiles, below which writing and joining the pieces costs more than it evens out.
  const long long all = s_tiles * a.h_kv;
  long long most = 1LL << 40;
  if ((long long)items * a.h_kv < 4LL * n_cta) {
    most = (all + 2 * n_cta - 1) / (2 * n_cta);
    if (most < 4) most = 4;
  }
  int n_work = 0, n_slot = 0, n_join = 0;
  for (int c0 = 0; c0 < items; c0 += kPlanThreads) {
    const int i = c0 + tid;
    int r = 0, tok0 = 0, nt = 0, pieces = 0;
    if (i < items) {
      r = find(i, &tok0);
      nt = item_tiles(a, load_chunk(a, r), tok0, tpi);
      pieces = nt <= most ? 1 : (int)((nt + most - 1) / most);
    }
    int t_work, t_slot, t_join;
    const int w = n_work + block_scan(pieces, s_warp, &t_work);
    const int s = n_slot + block_scan(pieces > 1 ? pieces : 0, s_warp, &t_slot);
    const int j = n_join + block_scan(pieces > 1 ? 1 : 0, s_warp, &t_join);
    for (int q = 0; q < pieces; ++q) {
      ChunkWork x;
      x.r = r;
      x.tok0 = tok0;
      // equal pieces rather than full ones and a remainder
      x.t0 = (int)((long long)q * nt / pieces);
      x.t1 = (int)((long long)(q + 1) * nt / pieces);
      x.slot = pieces > 1 ? s + q : -1;
      x.pad[0] = x.pad[1] = x.pad[2] = 0;
      k.ws.work[w + q] = x;
    }
    if (pieces > 1) {
      ChunkJoin x;
      x.r = r;
      x.tok0 = tok0;
      x.slot = s;
      x.n = pieces;
      k.ws.joins[j] = x;
    }
    n_work += t_work;
    n_slot += t_slot;
    n_join += t_join;
  }
  if (tid == 0) {
    ChunkHead h;
    h.n_work = n_work;
    h.n_join = n_join;
    h.slots_per_head = n_slot;
    h.pad = 0;
    *k.ws.head = h;
  }
}

// Shared-memory descriptor of a B operand whose N dimension is contiguous: rows are keys of 128 bytes
// (64 channels), groups of 8 rows 1024 bytes apart, the other 64 channels one k-block further.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(kKBlock >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void mma_pv(uint32_t tmem_o, uint32_t tmem_p, uint32_t v_addr, uint32_t idesc, bool accumulate) {
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const uint64_t db = desc_mn(v_addr + ks * 16 * 128);
    const uint32_t acc = (accumulate || ks > 0) ? 1u : 0u;
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n}\n" ::"r"(tmem_o),
        "r"(tmem_p + 8u * ks), "l"(db), "r"(idesc), "r"(acc), "r"(0u)
        : "memory");
  }
}
__device__ __forceinline__ void tmem_st32(const uint32_t* r, uint32_t taddr) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_ld8(float* v, uint32_t taddr) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void tmem_st8(const float* v, uint32_t taddr) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// Q rows of one tile half: (64 channels, G heads, tokens, batch row) boxes.
__device__ __forceinline__ void q_copy(const CUtensorMap* map, uint32_t dst, uint64_t* bar, int kb, int head, int tok, int b) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(kb * 64), "r"(head), "r"(tok), "r"(b), "r"(zc_smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void expect_bytes(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(zc_smem_u32(bar)), "r"(bytes) : "memory");
}

// An item as every role of a CTA derives it from the list.
struct Item {
  int r, kv, tok0, ntok;      // request (dense form: batch row), KV head, tokens
  int row0;                   // row of the request's token 0
  int p_first;
  int t0, t1, slot;
  ZcSeen s;
  int ga[2], ge[2];           // key tiles that group 0 / 1 takes part in (empty: ga >= ge)
  __device__ __forceinline__ int key0(int t) const { return (t < s.nsb ? t : s.wb0 + t - s.nsb) << kTileLog2; }
};

template <bool PAGED>
__device__ __forceinline__ Item load_item(const ChunkArgs& k, long long idx, int n_work) {
  const ZcPagedArgs& a = k.a;
  Item it;
  const int tpi = 2 * k.tpt;
  int n;
  if (PAGED) {
    it.kv = (int)(idx / n_work);
    const ChunkWork w = k.ws.work[idx - (long long)it.kv * n_work];
    const Chunk c = load_chunk(a, w.r);
    it.r = w.r;
    it.tok0 = w.tok0;
    it.t0 = w.t0;
    it.t1 = w.t1;
    it.slot = w.slot;
    it.row0 = c.row0;
    it.p_first = c.p0 + w.tok0;
    n = c.n;
  } else {
    const int unit = (int)(idx / k.items);
    it.r = unit / a.h_kv;
    it.kv = unit - it.r * a.h_kv;
    it.tok0 = (k.items - 1 - (int)(idx - (long long)unit * k.items)) * tpi;   // the last, longest rows first
    it.slot = -1;
    it.row0 = 0;
    it.p_first = it.tok0;
    n = k.l;
  }
  it.ntok = min(tpi, n - it.tok0);
  it.s = zc_seen(it.p_first, it.p_first + it.ntok - 1, a.window, a.sinks, kTileLog2);
  if (!PAGED) {
    it.t0 = 0;
    it.t1 = it.s.nb;
  }
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int first = it.p_first + g * k.tpt, last = it.p_first + min(it.ntok, (g + 1) * k.tpt) - 1;
    const int lo = max(0, first - a.window + 1), hi = max(0, last + 1);
    const int end = it.s.nsb + max(0, ((hi + kM - 1) >> kTileLog2) - it.s.wb0);
    const int begin = it.s.nsb > 0 ? 0 : max(0, (lo >> kTileLog2) - it.s.wb0);
    it.ga[g] = max(it.t0, begin);
    it.ge[g] = last >= first ? min(it.t1, end) : it.t0;
  }
  return it;
}

template <typename T, bool PAGED>
__global__ void __launch_bounds__(kThreads, 1)
    k_chunk_attention(const ChunkArgs k, const __grid_constant__ CUtensorMap qmap,
                      const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  const ZcPagedArgs& a = k.a;
  const uint32_t raw_u = zc_smem_u32(smem_raw);
  const uint32_t base_u = (raw_u + 1023u) & ~1023u;
  char* base = smem_raw + (base_u - raw_u);
  const uint32_t q_addr = base_u, k_addr = base_u + 2 * kTile, v_addr = k_addr + kKS * kTile;
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + kTiles);
  uint64_t* q_full = bars;                  // an item's Q tiles landed
  uint64_t* q_free = bars + 1;              // an item's last S completed
  uint64_t* k_full = bars + 2;              // [kKS] key tile landed
  uint64_t* k_free = k_full + kKS;          // [kKS] both groups' S of that tile completed
  uint64_t* v_full = k_free + kKS;          // [kVS] value tile landed
  uint64_t* v_free = v_full + kVS;          // [kVS] both groups' P V of that tile completed
  uint64_t* s_done = v_free + kVS;          // [2] S_g of a tile completed
  uint64_t* p_full = s_done + 2;            // [2] the group's four warps have written P_g
  uint64_t* o_done = p_full + 2;            // [2] the group's last P V of an item completed
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_done + 2);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  if (tid == 0) {
    bar_init(q_full, 1);
    bar_init(q_free, 1);
    for (int i = 0; i < kKS; ++i) {
      bar_init(&k_full[i], 1);
      bar_init(&k_free[i], 1);
    }
    for (int i = 0; i < kVS; ++i) {
      bar_init(&v_full[i], 1);
      bar_init(&v_free[i], 1);
    }
    for (int g = 0; g < 2; ++g) {
      bar_init(&s_done[g], 1);
      bar_init(&p_full[g], 4);
      bar_init(&o_done[g], 1);
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
  asm volatile("griddepcontrol.wait;\n" ::: "memory");   // the list of work (and all that came before it)

  const int n_work = PAGED ? k.ws.head->n_work : k.items;
  const long long n_idx = PAGED ? (long long)n_work * a.h_kv : (long long)k.items * a.n_req * a.h_kv;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
    if (warp == 1) {
      // ---- copies ----
      uint32_t tile = 0, item = 0;   // key tiles and items (with tiles) so far
      for (long long idx = blockIdx.x; idx < n_idx; idx += gridDim.x) {
        const Item it = load_item<PAGED>(k, idx, n_work);
        if (it.t0 >= it.t1) continue;
        if (lane == 0) {
          if (item > 0) bar_wait(q_free, (item - 1) & 1u);
          const int tiles = it.ntok > k.tpt ? 2 : 1;
          expect_bytes(q_full, (uint32_t)(tiles * k.tpt * a.G * ZC_D * 2));
          for (int g = 0; g < tiles; ++g)
            for (int kb = 0; kb < 2; ++kb)
              q_copy(&qmap, q_addr + g * kTile + kb * kKBlock, q_full, kb, it.kv * a.G,
                     it.row0 + it.tok0 + g * k.tpt, PAGED ? 0 : it.r);
        }
        ++item;
        for (int t = it.t0; t < it.t1; ++t, ++tile) {
          const int ks = tile % kKS, vs = tile % kVS, key0 = it.key0(t);
          if (PAGED) {
            // lane i brings the i-th page of the tile, if any row of the item sees a key of it
            const int rows = min(kM, 1 << a.page_log2), n_page = kM / rows;
            const int pk0 = key0 + lane * rows;
            const bool on = lane < n_page &&
                            (pk0 < it.s.sink_n || (pk0 < it.s.hi && pk0 + rows > it.s.lo));
            const int page = on ? a.table[(long long)it.r * a.table_width + (pk0 >> a.page_log2)] : 0;
            const int pg = page >= 0 && page < a.n_pages ? page : a.n_pages;   // beyond the pool: arrives as zeros
            const int row = pk0 & ((1 << a.page_log2) - 1);
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, on)) * (uint32_t)rows * (ZC_D * 2);
            if (lane == 0) {
              if (tile >= kKS) bar_wait(&k_free[ks], (tile / kKS - 1) & 1u);
              expect_bytes(&k_full[ks], bytes);
            }
            __syncwarp();
            if (on)
              for (int kb = 0; kb < 2; ++kb)
                page_copy(&kmap, k_addr + ks * kTile + kb * kKBlock + lane * rows * 128, &k_full[ks], row, kb, it.kv, pg);
            if (lane == 0) {
              if (tile >= kVS) bar_wait(&v_free[vs], (tile / kVS - 1) & 1u);
              expect_bytes(&v_full[vs], bytes);
            }
            __syncwarp();
            if (on)
              for (int kb = 0; kb < 2; ++kb)
                page_copy(&vmap, v_addr + vs * kTile + kb * kKBlock + lane * rows * 128, &v_full[vs], row, kb, it.kv, pg);
          } else if (lane == 0) {
            if (tile >= kKS) bar_wait(&k_free[ks], (tile / kKS - 1) & 1u);
            tma_key_tile(&kmap, k_addr + ks * kTile, &k_full[ks], key0, it.kv, it.r);
            if (tile >= kVS) bar_wait(&v_free[vs], (tile / kVS - 1) & 1u);
            tma_key_tile(&vmap, v_addr + vs * kTile, &v_full[vs], key0, it.kv, it.r);
          }
        }
      }
    } else if (warp == 0 && lane == 0) {
      // ---- matrix products ----
      const uint32_t idesc_s = instr_desc<T>();
      const uint32_t idesc_pv = instr_desc<T>() | (1u << 16);   // B with its N dimension contiguous
      uint32_t tile = 0, item = 0, n_s[2] = {0, 0};             // n_s: S tiles of a group whose P V is issued
      for (long long idx = blockIdx.x; idx < n_idx; idx += gridDim.x) {
        const Item it = load_item<PAGED>(k, idx, n_work);
        if (it.t0 >= it.t1) continue;
        bar_wait(q_full, item & 1u);
        ++item;
        bar_wait(&k_full[tile % kKS], (tile / kKS) & 1u);
#pragma unroll
        for (int g = 0; g < 2; ++g)
          if (it.ga[g] == it.t0 && it.ga[g] < it.ge[g]) {
            mma_tile(tmem + g * kM, q_addr + g * kTile, k_addr + (tile % kKS) * kTile, idesc_s);
            mma_commit(&s_done[g]);
          }
        mma_commit(&k_free[tile % kKS]);
        if (it.t0 + 1 == it.t1) mma_commit(q_free);
        for (int t = it.t0; t < it.t1; ++t, ++tile) {
          const uint32_t vs = tile % kVS, next = tile + 1, ks1 = next % kKS;
          const uint32_t v_tile = v_addr + vs * kTile, k_next = k_addr + ks1 * kTile;
          bool v_ready = false, k_ready = false;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (t >= it.ga[g] && t < it.ge[g]) {
              bar_wait(&p_full[g], n_s[g] & 1u);
              ++n_s[g];
              if (!v_ready) bar_wait(&v_full[vs], (tile / kVS) & 1u);
              v_ready = true;
              tc_fence_after();
              mma_pv(tmem + (2 + g) * kM, tmem + g * kM, v_tile, idesc_pv, t > it.ga[g]);
              if (t + 1 == it.ge[g]) mma_commit(&o_done[g]);
            }
            if (t + 1 >= it.ga[g] && t + 1 < it.ge[g]) {
              if (!k_ready) bar_wait(&k_full[ks1], (next / kKS) & 1u);
              k_ready = true;
              tc_fence_after();
              mma_tile(tmem + g * kM, q_addr + g * kTile, k_next, idesc_s);
              mma_commit(&s_done[g]);
            }
          }
          mma_commit(&v_free[vs]);
          if (t + 1 < it.t1) {
            if (!k_ready) bar_wait(&k_full[ks1], (next / kKS) & 1u);
            mma_commit(&k_free[ks1]);
            if (t + 2 == it.t1) mma_commit(q_free);
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;\n");
    const int g = (warp >> 2) - 1, quarter = warp & 3, row = quarter * 32 + lane;
    const int tok_in = row / a.G, head_in = row - tok_in * a.G;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t tmem_s = tmem + lane_off + (uint32_t)g * kM, tmem_o = tmem + lane_off + (uint32_t)(2 + g) * kM;
    const float scale = kLog2e * rsqrtf((float)ZC_D);
    uint32_t tile0 = 0, n_s = 0, n_o = 0;
    for (long long idx = blockIdx.x; idx < n_idx; idx += gridDim.x) {
      const Item it = load_item<PAGED>(k, idx, n_work);
      const int tok = g * k.tpt + tok_in;                           // token of the item
      const bool valid = tok_in < k.tpt && tok < it.ntok;
      const int pos = valid ? it.p_first + tok : -1;
      const int first = it.p_first + g * k.tpt, last = it.p_first + min(it.ntok, (g + 1) * k.tpt) - 1;
      const int ga = g ? it.ga[1] : it.ga[0], ge = g ? it.ge[1] : it.ge[0];
      float m_run = kNoMax, s_run = 0.f;
      for (int t = ga; t < ge; ++t) {
        const int key0 = it.key0(t);
        float v[kM];
        bar_wait(&s_done[g], n_s & 1u);
        ++n_s;
        tc_fence_after();
        tmem_ld128(v, tmem_s);
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (key0 + kM - 1 > first || (key0 <= last - a.window && key0 + kM > a.sinks)) {
          // the tile crosses the diagonal, the window's edge or the end of the sinks
          const int e_hi = pos - key0, e_lo = max(pos - a.window, -1) - key0, e_sink = a.sinks - key0;
#pragma unroll
          for (int e = 0; e < kM; ++e) {
            if (!(e <= e_hi && (e > e_lo || e < e_sink))) v[e] = -INFINITY;
            mx4[e & 3] = fmaxf(mx4[e & 3], v[e]);
          }
          // values that no row of the item sees may hold anything (a weight of 0 times NaN is NaN)
          if (key0 + kM > it.s.hi || (key0 < it.s.lo && key0 + kM > it.s.sink_n)) {
            const uint32_t tile = tile0 + (uint32_t)(t - it.t0), vs = tile % kVS;
            bar_wait(&v_full[vs], (tile / kVS) & 1u);
            const int key = key0 + row;
            if (key >= it.s.hi || (key < it.s.lo && key >= it.s.sink_n)) {
              char* at = base + (v_addr - base_u) + vs * kTile + row * 128;
#pragma unroll
              for (int c = 0; c < 16; ++c)
                *reinterpret_cast<uint4*>(at + (c >> 3) * kKBlock + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            async_proxy_fence();
          }
        } else {
#pragma unroll
          for (int e = 0; e < kM; ++e) mx4[e & 3] = fmaxf(mx4[e & 3], v[e]);
        }
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale;
        const bool grow = mx > m_run + kTau;
        if (__any_sync(0xffffffffu, grow && t > ga)) {
          const float alpha = grow ? zc_exp2(m_run - mx) : 1.f;
#pragma unroll 1
          for (int q8 = 0; q8 < 16; ++q8) {
            float o[8];
            tmem_ld8(o, tmem_o + 8 * q8);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= alpha;
            tmem_st8(o, tmem_o + 8 * q8);
          }
        }
        if (grow) {
          s_run *= zc_exp2(m_run - mx);
          m_run = mx;
        }
        float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t w[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            const float p0 = zc_exp2(fmaf(v[64 * half + 2 * c], scale, -m_run));
            const float p1 = zc_exp2(fmaf(v[64 * half + 2 * c + 1], scale, -m_run));
            add[c & 1] += p0;
            add[2 + (c & 1)] += p1;
            w[c] = pack2<T>(p0, p1);
          }
          tmem_st32(w, tmem_s + 32 * half);
        }
        s_run += (add[0] + add[1]) + (add[2] + add[3]);
        asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(&p_full[g]);
      }
      tile0 += (uint32_t)max(0, it.t1 - it.t0);
      // ---- the row's output and log-sum-exp, or its partial result ----
      const bool any = ga < ge;
      if (any) {
        bar_wait(&o_done[g], n_o & 1u);
        ++n_o;
        tc_fence_after();
      }
      const int h = it.kv * a.G + head_in;
      if (it.slot < 0) {
        const bool some = any && s_run > 0.f;
        const float inv = some ? 1.f / s_run : 0.f;
        const long long at = (PAGED ? 0 : it.r * k.o_req) + (long long)(it.row0 + it.tok0 + tok) * k.o_row + h * k.o_head;
        T* orow = reinterpret_cast<T*>(a.out) + at;
#pragma unroll 1
        for (int q4 = 0; q4 < 4; ++q4) {
          float o[32];
          if (any) {
            tmem_ld32_nowait(o, tmem_o + 32 * q4);
            asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          }
          if (valid) {
#pragma unroll
            for (int c4 = 0; c4 < 4; ++c4) {
              uint4 w = make_uint4(pack2<T>(o[8 * c4] * inv, o[8 * c4 + 1] * inv),
                                   pack2<T>(o[8 * c4 + 2] * inv, o[8 * c4 + 3] * inv),
                                   pack2<T>(o[8 * c4 + 4] * inv, o[8 * c4 + 5] * inv),
                                   pack2<T>(o[8 * c4 + 6] * inv, o[8 * c4 + 7] * inv));
              if (!some) w = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(orow + 32 * q4 + 8 * c4) = w;
            }
          }
        }
        if (valid && a.lse) a.lse[at / ZC_D] = some ? m_run + log2f(s_run) : -INFINITY;
      } else {
        float* pr = k.ws.parts + (((long long)it.kv * k.ws.head->slots_per_head + it.slot) * kItemRows + g * kM + row) *
                                     kPartStride;
        if (valid) *reinterpret_cast<float4*>(pr) = make_float4(m_run, any ? s_run : 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int q4 = 0; q4 < 4; ++q4) {
          float o[32];
          if (any) {
            tmem_ld32_nowait(o, tmem_o + 32 * q4);
            asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (valid) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
              *reinterpret_cast<float4*>(pr + 4 + 32 * q4 + 4 * c) =
                  make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
          }
        }
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

// Rows of the items that were worked on in pieces: a warp per row.
template <typename T> __global__ void __launch_bounds__(256) k_chunk_join(const ChunkArgs k) {
  asm volatile("griddepcontrol.wait;\n" ::: "memory");
  const ZcPagedArgs& a = k.a;
  const ChunkHead hd = *k.ws.head;
  const int lane = threadIdx.x & 31;
  const long long n = (long long)hd.n_join * a.h_kv * kItemRows;
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) >> 5; i < n; i += (long long)gridDim.x * 8) {
    const int row = (int)(i % kItemRows), g = row / kM, in = row % kM;
    const long long job = i / kItemRows;
    const int kv = (int)(job / hd.n_join);
    const ChunkJoin j = k.ws.joins[job - (long long)kv * hd.n_join];
    const Chunk c = load_chunk(a, j.r);
    const int tok_in = in / a.G, tok = j.tok0 + g * k.tpt + tok_in;
    if (tok_in >= k.tpt || tok >= c.n) continue;
    const long long at = (long long)(c.row0 + tok) * a.h_q + kv * a.G + (in - tok_in * a.G);
    join_row<T>(a.out, a.lse, at, lane, j.n, [&](int q) {
      return k.ws.parts + (((long long)kv * hd.slots_per_head + j.slot + q) * kItemRows + row) * kPartStride;
    });
  }
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
int tokens_per_tile(int G) { return kM / G; }

// Places of the parts of a call's workspace; returns the bytes.
size_t carve(char* ws, int G, int h_kv, int n_req, int n_rows, ChunkWs* out) {
  const size_t items = (size_t)n_rows / (2 * tokens_per_tile(G)) + (size_t)n_req + 1;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = ws + off;
    off += round_up(bytes);
    return p;
  };
  ChunkWs w;
  w.head = (ChunkHead*)take(sizeof(ChunkHead));
  w.item_start = (int*)take(((size_t)n_req + 1) * sizeof(int));
  w.work = (ChunkWork*)take((items + kMaxSlots) * sizeof(ChunkWork));
  w.joins = (ChunkJoin*)take((size_t)kMaxSlots * sizeof(ChunkJoin));
  w.parts = (float*)take((size_t)kMaxSlots * kItemRows * kPartStride * sizeof(float));
  (void)h_kv;
  if (out) *out = w;
  return off;
}

template <typename T, bool PAGED>
cudaError_t ready() {   // the shared memory the kernel asks for, once per device
  static bool once[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && once[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(k_chunk_attention<T, PAGED>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e == cudaSuccess && dev >= 0 && dev < 64) once[dev] = true;
  return e;
}

// Q as (channels, query heads, tokens, batch rows), boxes of 64 channels x G heads x tpt tokens.
bool make_q_map(CUtensorMap* map, const void* q, int dtype, int h_q, int G, long long tokens, int batch,
                long long s_head, long long s_tok, long long s_batch) {
  const cuuint64_t dims[4] = {ZC_D, (cuuint64_t)h_q, (cuuint64_t)tokens, (cuuint64_t)batch};
  // an extent of 1 may come with any stride: the map wants one that is valid
  const long long s[3] = {h_q > 1 ? s_head : ZC_D, tokens > 1 ? s_tok : ZC_D, batch > 1 ? s_batch : ZC_D};
  cuuint64_t strides[3];
  for (int i = 0; i < 3; ++i) {
    if (s[i] <= 0 || (s[i] & 7)) return false;
    strides[i] = (cuuint64_t)s[i] * 2;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)G, (cuuint32_t)tokens_per_tile(G), 1};
  return zc_encode_map(map, dtype, 4, q, dims, strides, box);
}

template <typename T>
int launch_chunk(zc_pages* p, const ChunkArgs& k, const CUtensorMap& qmap, cudaStream_t st) {
  cudaError_t e = ready<T, true>();
  if (e != cudaSuccess) return e;
  k_chunk_plan<<<1, kPlanThreads, 0, st>>>(k, p->n_sm);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  e = zc_launch_early(k_chunk_attention<T, true>, dim3(p->n_sm), dim3(kThreads), kSmem, st, k, qmap, p->k128, p->v128);
  if (e != cudaSuccess) return e;
  e = zc_launch_early(k_chunk_join<T>, dim3(2 * p->n_sm), dim3(256), 0, st, k);
  p->launches += 3;
  return e;
}

}  // namespace

size_t zc_paged_chunk_workspace(const zc_pages* p, int n_req, int n_rows) {
  return carve(nullptr, p->G, p->cfg.n_kv_heads, n_req, n_rows, nullptr);
}

int zc_launch_paged_chunk(zc_pages* p, const ZcPagedArgs& a, char* ws, cudaStream_t st) {
  if (!zc_page_maps(p)) return (int)cudaErrorNotSupported;
  ChunkArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  carve(ws, a.G, a.h_kv, a.n_req, a.n_rows, &k.ws);
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
      !make_key_map(&kmap, K, cfg.dtype, l, cfg.n_kv_heads, cfg.batch, ks) ||
      !make_key_map(&vmap, V, cfg.dtype, l, cfg.n_kv_heads, cfg.batch, ks))
    return (int)cudaErrorNotSupported;
  const long long n = (long long)k.items * cfg.batch * cfg.n_kv_heads;
  const int grid = n < c->n_sm ? (int)n : c->n_sm;
  cudaError_t e;
  if (cfg.dtype == ZC_F16) {
    e = ready<__half, false>();
    if (e != cudaSuccess) return e;
    k_chunk_attention<__half, false><<<grid, kThreads, kSmem, st>>>(k, qmap, kmap, vmap);
  } else {
    e = ready<__nv_bfloat16, false>();
    if (e != cudaSuccess) return e;
    k_chunk_attention<__nv_bfloat16, false><<<grid, kThreads, kSmem, st>>>(k, qmap, kmap, vmap);
  }
  c->launches += 1;
  return (int)cudaGetLastError();
}

int zc_paged_chunk_error_code(int* out) { return (int)cudaMemcpyFromSymbol(out, g_zc_tc_error, sizeof(int)); }
