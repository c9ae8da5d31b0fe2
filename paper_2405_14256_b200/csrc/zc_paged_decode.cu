// Attention of a few rows per request (a generated token, or a handful: rows x query heads of a KV
// head <= 16) over its cached keys in pages (Eq. 4; bound: HBM, every visible key and value once).
//
// The visible keys of every (request, KV head) are cut into steps of 128 (eight blocks of 16); all
// steps of the call, laid end to end, are dealt out to the CTAs in equal, consecutive shares, so that
// ragged lengths do not matter (units of a few steps stay whole).  A CTA is eight warps; warp w takes block w
// of each step through a ring of its own (bulk tensor copies of 16 keys and 16 values, 8 KB a stage), so that
// no warp waits for another inside a share.  Per block, with the query rows as the N dimension of the tensor-core tiles:
//   S^T (16 keys x 8 rows) = K Q^T        A = keys from shared memory, B = rows kept in registers
//   O^T (128 x 8 rows)    += V^T P^T      A = values read transposed, B = P^T = 2^(S - m), transposed in registers,
//                                         in two parts of the input type: the weight rounded, and the rest of it, so that
//                                         the output is off by its own rounding alone (bf16, relative in norm: 0.0016,
//                                         with the rounded weight alone 0.0022).  The second products cost 0.5 % of a
//                                         large call and 0.25 us of a short one: the tensor cores have little else to do.
// Running maximum and sum per row in fp32; O is rescaled only when a row's maximum grows by more than
// 8 (base 2).  At the end of a unit's steps the eight warps' results meet in shared memory.  A unit
// that one CTA holds whole is written out; the pieces of one that a share's border cuts go to the workspace,
// and the CTA that brings the last of them puts them together, in the order of the CTAs (the result does not
// depend on timing).  It knows by a counter per unit, zero before and after every call.
//   32 requests of 2048-4096 tokens, 32 KV heads: 219-224 us, 6.7 TB/s; a window of 4096 over 16 requests, 8 KV heads:
// 48.2 us, 5.6 TB/s; 4 requests of 200-512 tokens: 7.6 us, of which launch, lengths and tables, one round trip to the
// keys and the join are all.
#include <cstring>
#include "zc_paged_block.cuh"

namespace {

constexpr int kDecWarps = 8, kDecThreads = 32 * kDecWarps;
constexpr int kStages = 2;                              // 3 measured 229 against 216 us (32 x 2048-4096 tokens, 32 KV heads)
constexpr int kRing = kDecWarps * kStages * 2 * kHalf;  // 128 KB
constexpr int kJoinStride = ZC_PART_STRIDE;            // m, sum, -, -, acc[128]
constexpr int kJoinBytes = kDecWarps * 8 * kJoinStride * 4;
constexpr int kScanBytes = kDecWarps * 8 + 2 * 80;    // warps' sums; the units of the share's two borders
constexpr int kDecSmem = kRing + kJoinBytes + kDecWarps * kStages * 8 + kScanBytes + 1024;   // 1 KB: alignment
// A cut costs a partial result, its announcement and a join, and a share that straddles two units pays most of it
// twice.  So units of up to 5 steps are never cut (32 requests of 300-500 tokens, 8 KV heads: 13.7 us, cut 16.5),
// and no piece is shorter than half a share or 3 steps (one request of 8000 tokens: 14.7 us, else 19.2).
constexpr int kWhole = 5;
constexpr int kLeast = 3;
static_assert(ZC_PAGED_MAX_CTAS * 4 <= ZC_PAGES_SYNC_BYTES, "a counter per CTA");
struct Req {
  int row0, n, p0;   // first row, rows, position of the first
  ZcSeen s;
};
__device__ __forceinline__ int load_req(const ZcPagedArgs& a, int r, Req* q) {
  const int e0 = min(max(a.row_start[r], 0), a.n_rows);
  const int e1 = min(max(a.row_start[r + 1], e0), a.n_rows);
  const long long cap = (long long)a.table_width << a.page_log2;
  const int kv = (int)min((long long)max(a.kv_len[r], 0), cap);
  q->row0 = e0;
  q->n = min(e1 - e0, a.max_rows);
  q->p0 = kv - (e1 - e0);
  q->s = zc_seen(q->p0, q->p0 + q->n - 1, a.window, a.sinks, kBlkLog2);
  return q->n > 0 ? max(1, (q->s.nb + kDecWarps - 1) / kDecWarps) : 0;
}

// A border between two shares: the unit (request, KV head) that it lies in, and the step it falls on, moved to the
// unit's start or end where the unit is too short to be cut.
struct Place {
  int r, steps, kv, step;
  long long unit0;   // the unit's first step among all
  Req q;
};
static_assert(sizeof(Place) <= 80, "two borders fit their place");
__device__ __forceinline__ int cut_step(long long off, int steps, int least) {
  if (steps <= kWhole) return 2 * off < steps ? 0 : steps;
  return off < least ? 0 : steps - off < least ? steps : (int)off;
}

// One unit's steps a .. b - 1 inside a CTA's share.
struct Seg {
  int r, kv, a, b, steps;
  long long left;   // steps of the share after this segment
  Req q;
};
__device__ __forceinline__ bool seg_next(const ZcPagedArgs& a, Seg& g) {
  if (g.left <= 0) return false;
  if (++g.kv == a.h_kv) {
    g.kv = 0;
    do {
      if (++g.r >= a.n_req) return false;
      g.steps = load_req(a, g.r, &g.q);
    } while (g.steps == 0);
  }
  g.a = 0;
  g.b = (int)min((long long)g.steps, g.left);
  g.left -= g.b;
  return true;
}

// NT: groups of 8 rows.  WEIGHTS: the logits are kept for zc_launch_score_add.
template <typename T, int NT, bool WEIGHTS>
__global__ void __launch_bounds__(kDecThreads, 1)
    k_paged_decode(const ZcPagedArgs a, float* logits, float* __restrict__ parts, unsigned* __restrict__ arrived,
                   const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  extern __shared__ __align__(1024) char smem_raw[];
  const uint32_t raw_u = zc_smem_u32(smem_raw);
  const uint32_t base_u = (raw_u + 1023u) & ~1023u;
  char* base = smem_raw + (base_u - raw_u);
  float* s_join = reinterpret_cast<float*>(base + kRing);
  uint64_t* bars = reinterpret_cast<uint64_t*>(base + kRing + kJoinBytes);
  long long* s_sum = reinterpret_cast<long long*>(bars + kDecWarps * kStages);
  Place* s_place = reinterpret_cast<Place*>(s_sum + kDecWarps);   // [2] where the share begins, where it ends
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid < kDecWarps * kStages) bar_init(&bars[tid], 1);
  if (tid == 64) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&kmap)));
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&vmap)));
  }
  asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  // (what adds the weights up reads the lengths and old scores before it waits for this kernel: it may start only once what
  // came before is complete)
  if (!WEIGHTS) zc_let_next_start();
  zc_wait_for_last();
  if (WEIGHTS) zc_let_next_start();

  // ---- this CTA's share ----
  long long sum = 0;
  int mine = 0;   // steps of this thread's request (of the last one, where there are more requests than threads)
  Req mq;
  for (int r = tid; r < a.n_req; r += kDecThreads) {
    mine = load_req(a, r, &mq);
    sum += mine;
  }
  long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) s_sum[warp] = incl;
  __syncthreads();
  long long total = 0, off = incl - sum;   // off: steps of the requests before this thread's (if it has one)
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) off += s_sum[w];
    total += s_sum[w];
  }
  total *= a.h_kv;
  const int g = (int)min((long long)gridDim.x, total);   // shares; no two borders on the same step
  const int c = blockIdx.x;
  if (c >= g) return;
  const int least = total >= (long long)g * 2 * kLeast ? kLeast : max(1, (int)((total + g) / (2 * g)));
  const long long border[2] = {zc_muldiv(c, total, g), zc_muldiv(c + 1, total, g)};
  auto found = [&](int r) {   // this thread's request, if a border lies in it
    if (mine <= 0) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const long long in = border[i] - off * a.h_kv;
      if (in < 0 || in >= (long long)mine * a.h_kv) continue;
      Place p;
      p.r = r;
      p.steps = mine;
      p.kv = in < (1LL << 31) ? (int)((uint32_t)in / (uint32_t)mine) : (int)(in / mine);
      const long long in_unit = in - (long long)p.kv * mine;
      p.unit0 = border[i] - in_unit;
      p.step = cut_step(in_unit, mine, least);
      p.q = mq;
      s_place[i] = p;
    }
  };
  if (tid == 0 && c + 1 == g) {   // the last share ends behind the last unit
    s_place[1].unit0 = total;
    s_place[1].step = 0;
  }
  if (a.n_req <= kDecThreads) {
    found(tid);
  } else {
    long long before = 0;
    for (int c0 = 0; c0 < a.n_req; c0 += kDecThreads) {
      mine = c0 + tid < a.n_req ? load_req(a, c0 + tid, &mq) : 0;
      incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
      }
      __syncthreads();
      if (lane == 31) s_sum[warp] = incl;
      __syncthreads();
      off = before + incl - mine;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        if (w < warp) off += s_sum[w];
        before += s_sum[w];
      }
      found(c0 + tid);
      if (border[1] < before * a.h_kv) break;   // the same for all threads
    }
  }
  __syncthreads();
  long long unit0 = s_place[0].unit0;   // of the segment's unit: its first step among all
  Seg seg;
  seg.r = s_place[0].r;
  seg.kv = s_place[0].kv;
  seg.steps = s_place[0].steps;
  seg.q = s_place[0].q;
  seg.a = s_place[0].step;
  const long long begin = unit0 + seg.a, end = s_place[1].unit0 + s_place[1].step;
  if (begin >= end) return;
  if (seg.a == seg.steps) {   // the border was moved to the unit's end: the share begins with the next unit
    unit0 += seg.steps;
    seg.left = end - begin;
    seg_next(a, seg);
  } else {
    seg.b = (int)min((long long)seg.steps, seg.a + (end - begin));
    seg.left = (end - begin) - (seg.b - seg.a);
  }

  // ---- copies: lane 0 of every warp, running ahead of the warp's own blocks ----
  Seg ps = seg;
  int pstep = seg.a, pkey = -1, ppage = 0, pkv = 0;
  auto fetch = [&]() {   // the next block of this warp; its page id is asked for now and used at the next issue
    for (;;) {
      for (; pstep < ps.b; ++pstep) {
        const int vb = pstep * kDecWarps + warp;
        if (vb < ps.q.s.nb) {
          pkey = (vb < ps.q.s.nsb ? vb : ps.q.s.wb0 + vb - ps.q.s.nsb) << kBlkLog2;
          pkv = ps.kv;
          ppage = a.table[(long long)ps.r * a.table_width + (pkey >> a.page_log2)];
          ++pstep;
          return;
        }
      }
      if (!seg_next(a, ps)) {
        pkey = -1;
        return;
      }
      pstep = 0;
    }
  };
  const uint32_t ring = base_u + warp * kStages * 2 * kHalf;
  uint64_t* full = bars + warp * kStages;
  bool ok = true;   // no wait of the warp has run out
  int held[2] = {0, 0};   // pages of the blocks in the two stages
  auto issue = [&](int stage) {
    if (pkey < 0) return;
    if (WEIGHTS) held[0] = stage == 0 ? ppage : held[0], held[1] = stage == 1 ? ppage : held[1];
    if (lane == 0) {
      const int page = ppage >= 0 && ppage < a.n_pages ? ppage : a.n_pages;   // beyond the pool: arrives as zeros
      const int row = pkey & ((1 << a.page_log2) - 1);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(zc_smem_u32(&full[stage])),
                   "r"(2 * kHalf)
                   : "memory");
      const uint32_t dst = ring + stage * 2 * kHalf;
      page_copy(&kmap, dst, &full[stage], row, 0, pkv, page);
      page_copy(&vmap, dst + kHalf, &full[stage], row, 0, pkv, page);
    }
    fetch();
  };
  fetch();
#pragma unroll
  for (int i = 0; i < kStages; ++i) issue(i);

  // The eight warps' results of the row that this warp takes, joined in their order.
  auto meet = [&](float& m, float& sum, float4& acc) {
    m = kNoMax;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) m = fmaxf(m, s_join[(w * 8 + warp) * kJoinStride]);
    sum = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      const float* jr = s_join + (w * 8 + warp) * kJoinStride;
      const float f = zc_exp2(jr[0] - m);
      const float4 x = *reinterpret_cast<const float4*>(jr + 4 + 4 * lane);
      sum = fmaf(jr[1], f, sum);
      acc.x = fmaf(x.x, f, acc.x);
      acc.y = fmaf(x.y, f, acc.y);
      acc.z = fmaf(x.z, f, acc.z);
      acc.w = fmaf(x.w, f, acc.w);
    }
  };
  const int quad = lane & 3, oct = lane >> 2;
  int stage = 0;
  uint32_t phase = 0;
  for (;;) {
    const int rows = seg.q.n * a.G;
    uint32_t qf[NT][8][2];
    int pos[NT][2];
    load_rows<T, NT>(a, seg.q.row0, seg.kv, rows, qf);
    row_positions<NT>(a, seg.q.p0, rows, pos);
    const int p_last = seg.q.p0 + seg.q.n - 1;
    RowState<NT> x;
    x.clear();
    for (int step = seg.a; ok && step < seg.b; ++step) {
      const int vb = step * kDecWarps + warp;
      if (vb >= seg.q.s.nb) break;
      const int key0 = (vb < seg.q.s.nsb ? vb : seg.q.s.wb0 + vb - seg.q.s.nsb) << kBlkLog2;
      const uint32_t kt = ring + stage * 2 * kHalf, vt = kt + kHalf;
      ok = warp_wait(&full[stage], phase);
      if (!ok) break;   // nothing more is copied; the unit's other warps are met below
      float* keep = nullptr;
      if (WEIGHTS) {
        const int page = stage == 0 ? held[0] : held[1];
        if (page >= 0 && page < a.n_pages) keep = logits_of(logits, a, page, seg.kv, key0);
      }
      attend_block<T, NT, WEIGHTS>(x, qf, pos, kt, vt, base + (vt - base_u), key0, seg.q.p0, p_last, seg.q.s, a, rows, keep);
      __syncwarp();
      issue(stage);
      if (++stage == kStages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    // ---- the eight warps' results of this unit ----
    const bool whole = seg.a == 0 && seg.b == seg.steps;
    // (a CTA has one piece at most that does not begin with its unit, and one that does and does not end with it)
    float* slot = parts + (2 * c + (seg.a > 0 ? 0 : 1)) * (long long)ZC_PAGED_ROWS * kJoinStride;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (8 * nt >= rows) break;
      __syncthreads();   // the join area is free
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float t = x.s[nt][e];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) t += __shfl_xor_sync(0xffffffffu, t, x);
        float* jr = s_join + (warp * 8 + 2 * quad + e) * kJoinStride;
        if (oct == 0) {
          jr[0] = x.m[nt][e];
          jr[1] = t;
        }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) {
          jr[4 + 16 * mt + oct] = x.o[nt][mt][e];
          jr[4 + 16 * mt + oct + 8] = x.o[nt][mt][e + 2];
        }
      }
      __syncthreads();
      const int row = 8 * nt + warp;
      if (row < rows) {
        float mt, total_s;
        float4 acc;
        meet(mt, total_s, acc);
        if (whole) {
          const int tok = row / a.G;
          const long long at = (long long)(seg.q.row0 + tok) * a.h_q + seg.kv * a.G + (row - tok * a.G);
          store_row<T>(a.out, a.lse, at, lane, mt, total_s, acc);
        } else {
          float* pr = slot + row * kJoinStride;
          if (lane == 0) {
            pr[0] = mt;
            pr[1] = total_s;
          }
          *reinterpret_cast<float4*>(pr + 4 + 4 * lane) = acc;
        }
      }
    }
    if (!whole) {
      // The CTAs whose shares begin inside the unit; the one before the first of them has its first steps.
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        auto cuts = [&](int d) {
          if (d < 1 || d >= g) return false;
          const long long in = zc_muldiv(d, total, g) - unit0;
          if (in <= 0 || in >= seg.steps) return false;
          const int t = cut_step(in, seg.steps, least);
          return t > 0 && t < seg.steps;
        };
        int c0 = c, c1 = c;
        if (seg.a > 0)
          while (cuts(c0 - 1)) --c0;
        while (cuts(c1 + 1)) ++c1;
        if (seg.a > 0) --c0;
        s_place[0].r = c0;
        s_place[0].kv = c1;
        s_place[0].step = atomicAdd(&arrived[c0], 1u) == (unsigned)(c1 - c0);
      }
      __syncthreads();
      if (s_place[0].step) {
        __threadfence();
        const int c0 = s_place[0].r, n = s_place[0].kv - c0 + 1;
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
          // warp w takes pieces w, w + 8, ... of eight rows; then the warps' results meet as a unit's do
          __syncthreads();
          for (int r = 0; r < 8 && r0 + r < rows; r += 4) {
            float2 ms[4];
            float4 acc[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              ms[u] = make_float2(kNoMax, 0.f);
              acc[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            for (int i = warp; i < n; i += kDecWarps) {
              const float* pr = parts + ((long long)(2 * (c0 + i) + (i == 0 ? 1 : 0)) * ZC_PAGED_ROWS + r0 + r) * kJoinStride;
              float2 pm[4];
              float4 x[4];
#pragma unroll
              for (int u = 0; u < 4; ++u)
                if (r0 + r + u < rows) {
                  pm[u] = __ldcg(reinterpret_cast<const float2*>(pr + u * kJoinStride));
                  x[u] = __ldcg(reinterpret_cast<const float4*>(pr + u * kJoinStride + 4 + 4 * lane));
                }
#pragma unroll
              for (int u = 0; u < 4; ++u)
                if (r0 + r + u < rows) {
                  const float top = fmaxf(ms[u].x, pm[u].x), fo = zc_exp2(ms[u].x - top), fn = zc_exp2(pm[u].x - top);
                  ms[u] = make_float2(top, fmaf(ms[u].y, fo, pm[u].y * fn));
                  acc[u] = make_float4(fmaf(acc[u].x, fo, x[u].x * fn), fmaf(acc[u].y, fo, x[u].y * fn),
                                       fmaf(acc[u].z, fo, x[u].z * fn), fmaf(acc[u].w, fo, x[u].w * fn));
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              float* jr = s_join + (warp * 8 + r + u) * kJoinStride;
              if (lane == 0) {
                jr[0] = ms[u].x;
                jr[1] = ms[u].y;
              }
              *reinterpret_cast<float4*>(jr + 4 + 4 * lane) = acc[u];
            }
          }
          __syncthreads();
          const int row = r0 + warp;
          if (row < rows) {
            float m8, sum8;
            float4 acc8;
            meet(m8, sum8, acc8);
            const int tok = row / a.G;
            store_row<T>(a.out, a.lse, (long long)(seg.q.row0 + tok) * a.h_q + seg.kv * a.G + (row - tok * a.G), lane, m8, sum8, acc8);
          }
        }
        if (tid == 0) arrived[c0] = 0;   // as the next call wants it
      }
    }
    unit0 += seg.steps;
    if (!seg_next(a, seg)) break;
  }
  if (!ok)   // the copies that were on their way
    for (int i = 0; i < kStages; ++i) drain(&full[i], i < stage ? phase ^ 1u : phase);
}

template <typename T, int NT, bool WEIGHTS>
int launch(zc_pages* p, const ZcPagedArgs& a, float* logits, float* parts, unsigned* arrived, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed{0};
  cudaError_t e = zc_allow_smem(k_paged_decode<T, NT, WEIGHTS>, kDecSmem, &allowed);
  if (e != cudaSuccess) return e;
  e = zc_launch_early(k_paged_decode<T, NT, WEIGHTS>, dim3(p->n_sm), dim3(kDecThreads), kDecSmem, st, a, logits, parts, arrived,
                      p->k16, p->v16);
  if (e != cudaSuccess) return e;
  p->launches += 1;
  return cudaSuccess;
}

template <typename T, int NT>
int launch_mode(zc_pages* p, const ZcPagedArgs& a, float* logits, float* parts, unsigned* arrived, cudaStream_t st) {
  return logits ? launch<T, NT, true>(p, a, logits, parts, arrived, st) : launch<T, NT, false>(p, a, logits, parts, arrived, st);
}

}  // namespace

size_t zc_paged_decode_workspace() {
  return ZC_PAGES_SYNC_BYTES + (size_t)ZC_PAGED_MAX_CTAS * 2 * ZC_PAGED_ROWS * kJoinStride * 4;
}

int zc_launch_paged_decode(zc_pages* p, const ZcPagedArgs& a, float* logits, char* ws, cudaStream_t st) {
  if (!zc_page_maps(p)) return (int)cudaErrorNotSupported;
  unsigned* arrived = (unsigned*)ws;
  float* parts = (float*)(ws + ZC_PAGES_SYNC_BYTES);
  const bool one = a.max_rows * a.G <= 8;
  if (p->cfg.dtype == ZC_F16)
    return one ? launch_mode<__half, 1>(p, a, logits, parts, arrived, st) : launch_mode<__half, 2>(p, a, logits, parts, arrived, st);
  return one ? launch_mode<__nv_bfloat16, 1>(p, a, logits, parts, arrived, st)
             : launch_mode<__nv_bfloat16, 2>(p, a, logits, parts, arrived, st);
}

// Tensor maps of the pages: (64 channels, token of the page, half of the channels, KV head, page).
bool zc_page_maps(zc_pages* p) {
  if (p->maps_ready.load(std::memory_order_acquire)) return true;
  std::lock_guard<std::mutex> lock(p->maps_guard);
  if (p->maps_ready.load(std::memory_order_relaxed)) return true;   // another thread's first call
  const int64_t* s = p->cfg.strides;
  const cuuint64_t dims[5] = {64, (cuuint64_t)p->cfg.page_size, 2, (cuuint64_t)p->cfg.n_kv_heads,
                              (cuuint64_t)p->cfg.n_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)s[1] * 2, 128, (cuuint64_t)s[2] * 2, (cuuint64_t)s[0] * 2};
  const cuuint32_t small[5] = {64, kBlk, 2, 1, 1};
  // a tile of 64 keys from one page comes with both halves of its channels, from several pages half by half
  const bool one = p->cfg.page_size >= 64;
  const cuuint32_t large[5] = {64, (cuuint32_t)(one ? 64 : p->cfg.page_size), one ? 2u : 1u, 1, 1};
  const cuuint32_t tall[5] = {64, (cuuint32_t)(p->cfg.page_size < 128 ? p->cfg.page_size : 128), 1, 1, 1};
  struct { CUtensorMap* map; void* at; const cuuint32_t* box; } todo[5] = {
      {&p->k16, p->k, small}, {&p->v16, p->v, small}, {&p->k64, p->k, large}, {&p->v64, p->v, large}, {&p->k128, p->k, tall}};
  for (auto& t : todo)
    if (!zc_encode_map(t.map, p->cfg.dtype, 5, t.at, dims, strides, t.box)) return false;
  p->maps_ready.store(true, std::memory_order_release);
  return true;
}

int zc_paged_decode_error_code(int* out) { return (int)cudaMemcpyFromSymbol(out, g_zc_tc_error, sizeof(int)); }
