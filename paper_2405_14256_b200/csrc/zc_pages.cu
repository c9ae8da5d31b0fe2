// Full-precision pages: host API (argument checks, handle), block tables and slot maps from request
// lengths, and the copies between dense rows and pages.
#include <new>
#include "zc_paged.cuh"

namespace {

constexpr int kTabThreads = 256;
constexpr int kTabChunk = 4 * kTabThreads;   // requests one pass of the scan takes

__device__ __forceinline__ long long warp_incl(long long v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Block tables and slot maps.  Every CTA scans the lengths (two prefix sums, new rows and new pages,
// 1024 requests per pass) and then writes its share: requests and rows are dealt out in strides of
// the grid.  A row's page comes from the table where the request held it before, and straight from
// the free list where this call grants it, so no CTA waits for another's table entries.  Bound: latency, two
// round trips to memory and the scan: 2.6 us for 8 requests, 6.0 us for 1024 with 130000 rows.
__global__ void __launch_bounds__(kTabThreads) k_page_tables(
    int page_log2, int n_req, const int32_t* past, const int32_t* fresh, const int32_t* free_pages, int n_free,
    const int32_t* free_state,
    int32_t* table, int width, int32_t* __restrict__ kv_len, int32_t* __restrict__ row_start, int n_rows,
    int32_t* __restrict__ slots, int32_t* __restrict__ pos, int32_t* __restrict__ free_out) {
  __shared__ long long s_row[kTabChunk + 1], s_page[kTabChunk + 1];
  __shared__ int s_past[kTabChunk];
  __shared__ long long s_warp[3][kTabThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int psize = 1 << page_log2;
  zc_wait_for_last();
  const long long next = free_state[0] > 0 ? free_state[0] : 0;
  const long long end = free_state[1] < n_free ? free_state[1] : n_free;
  long long rows_before = 0, pages_before = 0, wanted = 0;
  for (int c0 = 0; c0 < n_req; c0 += kTabChunk) {
    // four consecutive requests per thread
    long long rows[4], pages[4], rsum = 0, psum = 0, want = 0;
    int pst[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = c0 + 4 * tid + i;
      const long long p = r < n_req && past[r] > 0 ? past[r] : 0, n = r < n_req && fresh[r] > 0 ? fresh[r] : 0;
      const long long had = (p + psize - 1) >> page_log2, has = (p + n + psize - 1) >> page_log2;
      const long long hadw = had < width ? had : width, hasw = has < width ? has : width;
      pst[i] = (int)p;
      rows[i] = rsum;
      pages[i] = psum;
      rsum += n;
      psum += hasw - hadw;
      want += has - had;
    }
    const long long ri = warp_incl(rsum, lane), pi = warp_incl(psum, lane), wi = warp_incl(want, lane);
    if (lane == 31) {
      s_warp[0][warp] = ri;
      s_warp[1][warp] = pi;
      s_warp[2][warp] = wi;
    }
    __syncthreads();
    long long ro = rows_before + ri - rsum, po = pages_before + pi - psum, rt = 0, pt = 0;
#pragma unroll
    for (int w = 0; w < kTabThreads / 32; ++w) {
      if (w < warp) {
        ro += s_warp[0][w];
        po += s_warp[1][w];
      }
      rt += s_warp[0][w];
      pt += s_warp[1][w];
      wanted += s_warp[2][w];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s_row[4 * tid + i] = ro + rows[i];
      s_page[4 * tid + i] = po + pages[i];
      s_past[4 * tid + i] = pst[i];
    }
    if (tid == 0) {
      s_row[kTabChunk] = rows_before + rt;
      s_page[kTabChunk] = pages_before + pt;
    }
    __syncthreads();
    const int here = min(kTabChunk, n_req - c0);
    // requests: a thread writes lengths, a warp the new table entries
    for (int i = blockIdx.x * kTabThreads + tid; i < here; i += gridDim.x * kTabThreads) {
      kv_len[c0 + i] = (int)(s_past[i] + s_row[i + 1] - s_row[i]);
      row_start[c0 + i] = (int)s_row[i];
    }
    for (int i = blockIdx.x * (kTabThreads / 32) + warp; i < here; i += gridDim.x * (kTabThreads / 32)) {
      const int had = (int)min((long long)width, ((long long)s_past[i] + psize - 1) >> page_log2);
      const long long n = s_page[i + 1] - s_page[i];
      for (long long k = lane; k < n; k += 32) {
        const long long at = next + s_page[i] + k;
        table[(long long)(c0 + i) * width + had + k] = at < end ? free_pages[at] : -1;
      }
    }
    // rows of these requests
    const long long row_end = min((long long)n_rows, rows_before + rt);
    for (long long row = rows_before + blockIdx.x * kTabThreads + tid; row < row_end;
         row += (long long)gridDim.x * kTabThreads) {
      int a = 0, b = here;   // the last request that starts at or before the row
      while (b - a > 1) {
        const int m = (a + b) >> 1;
        if (s_row[m] <= row) a = m; else b = m;
      }
      const long long p = (long long)s_past[a] + (row - s_row[a]);
      const long long idx = p >> page_log2;
      const long long had = ((long long)s_past[a] + psize - 1) >> page_log2;
      int page = -1;
      if (idx < width) {
        if (idx < had) page = table[(long long)(c0 + a) * width + idx];
        else {
          const long long at = next + s_page[a] + (idx - had);
          if (at < end) page = free_pages[at];
        }
      }
      pos[row] = (int)p;
      // (a page whose slots pass 31 bits is in no pool)
      const bool some = page >= 0 && page <= (0x7fffffff >> page_log2);
      slots[row] = some ? (page << page_log2) + (int)(p & (psize - 1)) : -1;
    }
    rows_before += rt;
    pages_before += pt;
    __syncthreads();
  }
  for (long long row = rows_before + blockIdx.x * kTabThreads + tid; row < n_rows;
       row += (long long)gridDim.x * kTabThreads) {
    pos[row] = -1;
    slots[row] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    row_start[n_req] = (int)rows_before;
    const long long room = end > next ? end - next : 0;
    const long long took = pages_before < room ? pages_before : room;
    free_out[0] = (int)(next + took);
    free_out[1] = (int)end;
    free_out[2] = (int)(wanted - took);
  }
}

// 16 lanes move the 256 bytes of one (row, head) of K and of V; a thread has kUnroll of them in
// flight.  Bound: HBM (each row read once and written once): 8 prompts of 4096 tokens, 8 KV heads, 40.5 us
// written and 43.0 us read back, 6.4 and 6.2 TB/s; 16 single tokens 2.6 us, the launch.
constexpr int kCopyThreads = 256, kUnroll = 4;

__global__ void __launch_bounds__(kCopyThreads) k_page_write(
    char* __restrict__ kp, char* __restrict__ vp, long long sp, long long st, long long sh, int page_log2,
    int n_pages, int h_kv, const char* kr, const char* vr, long long rs_row, long long rs_head,
    const int32_t* slots, long long n_pieces) {
  const int part = (threadIdx.x & 15) * 16, group = threadIdx.x >> 4;
  const long long first = ((long long)blockIdx.x * kUnroll) * (kCopyThreads / 16) + group;
  zc_let_next_start();
  zc_wait_for_last();
  uint4 k[kUnroll], v[kUnroll];
  char* kd[kUnroll];
  long long off[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const long long i = first + u * (kCopyThreads / 16);
    kd[u] = nullptr;
    if (i < n_pieces) {
      const long long row = i / h_kv;
      const int head = (int)(i - row * h_kv);
      const int slot = slots[row];
      if (slot >= 0 && (slot >> page_log2) < n_pages) {
        off[u] = (long long)(slot >> page_log2) * sp + (long long)(slot & ((1 << page_log2) - 1)) * st + head * sh + part;
        kd[u] = kp + off[u];
        const long long src = row * rs_row + head * rs_head + part;
        k[u] = *reinterpret_cast<const uint4*>(kr + src);
        v[u] = *reinterpret_cast<const uint4*>(vr + src);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (kd[u]) {
      *reinterpret_cast<uint4*>(kd[u]) = k[u];
      *reinterpret_cast<uint4*>(vp + off[u]) = v[u];
    }
}

// Block: (request, head) * blocks_per_head + block of 64 consecutive tokens of it.
__global__ void __launch_bounds__(kCopyThreads) k_page_read(
    const char* kp, const char* vp, long long sp, long long st, long long sh, int page_log2,
    int n_pages, int h_kv, const int32_t* table, int width, int l, char* __restrict__ K,
    char* __restrict__ V, long long ds_req, long long ds_head, long long ds_tok, int blocks_per_head) {
  const int part = (threadIdx.x & 15) * 16, group = threadIdx.x >> 4;
  const int unit = blockIdx.x / blocks_per_head, blk = blockIdx.x % blocks_per_head;
  const int r = unit / h_kv, head = unit % h_kv;
  const long long t0 = (long long)blk * kUnroll * (kCopyThreads / 16) + group;
  zc_let_next_start();
  zc_wait_for_last();
  uint4 k[kUnroll], v[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const long long t = t0 + u * (kCopyThreads / 16);
    k[u] = v[u] = make_uint4(0, 0, 0, 0);
    if (t < l) {
      const int idx = (int)(t >> page_log2);
      const int page = idx < width ? table[(long long)r * width + idx] : -1;
      if (page >= 0 && page < n_pages) {
        const long long off = (long long)page * sp + (t & ((1 << page_log2) - 1)) * st + head * sh + part;
        k[u] = *reinterpret_cast<const uint4*>(kp + off);
        v[u] = *reinterpret_cast<const uint4*>(vp + off);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const long long t = t0 + u * (kCopyThreads / 16);
    if (t < l) {
      const long long off = r * ds_req + head * ds_head + t * ds_tok + part;
      *reinterpret_cast<uint4*>(K + off) = k[u];
      *reinterpret_cast<uint4*>(V + off) = v[u];
    }
  }
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
template <typename... P> bool aligned4(const P*... p) { return (((uintptr_t)p | ...) & 3) == 0; }

struct Ints { const int32_t* at; long long n; };
bool overlap(const Ints& a, const Ints& b) { return a.n && b.n && a.at < b.at + b.n && b.at < a.at + a.n; }

int page_log2_of(int page_size) {
  for (int i = 4; i <= 8; ++i)
    if (page_size == 1 << i) return i;
  return -1;
}

int check_page_config(const zc_page_config* c) {
  if (!c || c->struct_size != (int)sizeof(zc_page_config)) return ZC_EINVAL;
  if (c->dtype != ZC_F16 && c->dtype != ZC_BF16) return ZC_EINVAL;
  if (c->n_kv_heads < 1 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads) return ZC_EINVAL;
  if (c->n_q_heads / c->n_kv_heads > ZC_PAGE_MAX_G || c->n_q_heads > 65535) return ZC_EINVAL;
  if (c->head_dim != ZC_D || page_log2_of(c->page_size) < 0 || c->reserved) return ZC_EINVAL;
  if (c->n_pages < 1 || (long long)c->n_pages * c->page_size > 0x7fffffffLL) return ZC_EINVAL;
  const long long extent[3] = {c->n_pages, c->page_size, c->n_kv_heads};
  for (int i = 0; i < 3; ++i) {
    // the tensor maps hold strides below 2^40 bytes
    if (c->strides[i] < 0 || c->strides[i] % 8 || c->strides[i] >= (1LL << 39)) return ZC_EINVAL;
    if (extent[i] > 1 && c->strides[i] < ZC_D) return ZC_EINVAL;
  }
  return ZC_OK;
}

// The checks that attention calls share, and what the kernels are given; n_req = 0 in *out: there is nothing to do.
int paged_args(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table, int table_width,
               const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows, int max_rows, int window, int sinks,
               void* out, float* row_lse, void* workspace, ZcPagedArgs* args) {
  args->n_req = 0;
  if (!p || !q_strides || n_req < 0 || n_rows < 0 || max_rows < 0 || window < 0 || sinks < 0) return ZC_EINVAL;
  if (n_req == 0 || n_rows == 0 || max_rows == 0) return ZC_OK;
  if (!q || !table || !row_start || !kv_len || !out || !workspace || table_width < 1) return ZC_EINVAL;
  if ((long long)table_width << p->page_log2 > ZC_NO_WINDOW || n_rows > ZC_NO_WINDOW) return ZC_EINVAL;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) || !aligned4(row_lse, table, row_start, kv_len))
    return ZC_EALIGN;
  for (int i = 0; i < 2; ++i)
    if (q_strides[i] < 0 || q_strides[i] % 8 || q_strides[i] >= (1LL << 39)) return ZC_EINVAL;
  if ((p->cfg.n_q_heads > 1 && q_strides[1] < ZC_D) || (n_rows > 1 && q_strides[0] < ZC_D)) return ZC_EINVAL;
  ZcPagedArgs& a = *args;
  a.table = table;
  a.row_start = row_start;
  a.kv_len = kv_len;
  a.table_width = table_width;
  a.n_req = n_req;
  a.n_rows = n_rows;
  a.max_rows = max_rows < n_rows ? max_rows : n_rows;
  a.page_log2 = p->page_log2;
  a.n_pages = p->cfg.n_pages;
  a.h_q = p->cfg.n_q_heads;
  a.h_kv = p->cfg.n_kv_heads;
  a.G = p->G;
  a.window = window == 0 || window > ZC_NO_WINDOW ? ZC_NO_WINDOW : window;
  a.sinks = sinks;
  a.q = q;
  a.qs_row = q_strides[0];
  a.qs_head = q_strides[1];
  a.out = out;
  a.lse = row_lse;
  return ZC_OK;
}
// Whether a call is the single-token kernel's.
bool few_rows(const ZcPagedArgs& a) { return (long long)a.max_rows * a.G <= ZC_PAGED_ROWS; }
// A logit of every slot, query head and row, where a call is.
size_t logits_bytes(const zc_page_config& c, int max_rows) {
  const int G = c.n_q_heads / c.n_kv_heads;
  return (long long)max_rows * G <= ZC_PAGED_ROWS ? (size_t)c.n_pages * c.page_size * c.n_q_heads * max_rows * 4 : 0;
}

}  // namespace

extern "C" {

int zc_pages_workspace(const zc_page_config* cfg, int n_req, int n_rows, size_t* workspace_bytes) {
  const int rc = check_page_config(cfg);
  if (rc) return rc;
  if (n_req < 0 || n_rows < 0 || !workspace_bytes) return ZC_EINVAL;
  if (!zc_paged_chunk_fits(cfg->n_q_heads / cfg->n_kv_heads, n_req, n_rows)) return ZC_ECAPACITY;
  const size_t a = zc_paged_decode_workspace(), b = zc_paged_chunk_workspace();
  *workspace_bytes = a > b ? a : b;
  return ZC_OK;
}

int zc_pages_init(void* k_pages, void* v_pages, const zc_page_config* cfg, zc_pages** out) {
  if (!out) return ZC_EINVAL;
  *out = nullptr;
  const int rc = check_page_config(cfg);
  if (rc) return rc;
  if (!k_pages || !v_pages) return ZC_EINVAL;
  if (!aligned16(k_pages) || !aligned16(v_pages)) return ZC_EALIGN;
  zc_pages* p = new (std::nothrow) zc_pages();
  if (!p) return ZC_EINVAL;
  p->cfg = *cfg;
  // an extent of 1 may come with any stride: the tensor maps want one that is valid
  const long long extent[3] = {cfg->n_pages, cfg->page_size, cfg->n_kv_heads};
  for (int i = 0; i < 3; ++i)
    if (extent[i] == 1) p->cfg.strides[i] = ZC_D;
  p->k = (char*)k_pages;
  p->v = (char*)v_pages;
  p->G = cfg->n_q_heads / cfg->n_kv_heads;
  p->page_log2 = page_log2_of(cfg->page_size);
  int dev = 0, n_sm = 148;
  if (cudaGetDevice(&dev) == cudaSuccess)
    cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev);
  else
    cudaGetLastError();
  p->n_sm = n_sm < 1 ? 148 : n_sm > ZC_PAGED_MAX_CTAS ? ZC_PAGED_MAX_CTAS : n_sm;
  *out = p;
  return ZC_OK;
}

void zc_pages_free(zc_pages* p) { delete p; }

int64_t zc_pages_launch_count(const zc_pages* p) { return p ? p->launches.load() : 0; }

int zc_page_tables(int page_size, int n_req, const int32_t* past, const int32_t* fresh, const int32_t* free_pages,
                   int n_free, const int32_t* free_state, int32_t* table, int table_width, int32_t* kv_len,
                   int32_t* row_start, int n_rows, int32_t* slots, int32_t* pos, int32_t* free_out,
                   zc_stream_t stream) {
  const int log2 = page_log2_of(page_size);
  if (log2 < 0 || n_req < 1 || n_rows < 0 || n_free < 0 || table_width < 1) return ZC_EINVAL;
  if ((long long)table_width << log2 > ZC_NO_WINDOW) return ZC_EINVAL;
  if (!past || !fresh || !free_state || !table || !kv_len || !row_start || !free_out) return ZC_EINVAL;
  if ((n_free && !free_pages) || (n_rows && (!slots || !pos))) return ZC_EINVAL;
  if (!aligned4(past, fresh, free_pages, free_state, table, kv_len, row_start, slots, pos, free_out)) return ZC_EALIGN;
  // every CTA reads all lengths, some after others have written their results
  const Ints in[4] = {{past, n_req}, {fresh, n_req}, {free_pages, n_free}, {free_state, 3}};
  const Ints out[6] = {{table, (long long)n_req * table_width}, {kv_len, n_req}, {row_start, n_req + 1LL},
                       {slots, n_rows}, {pos, n_rows}, {free_out, 3}};
  for (const Ints& i : in)
    for (const Ints& o : out)
      if (overlap(i, o)) return ZC_EINVAL;
  // a CTA per 1024 rows or 64 requests, whichever asks for more; at most two per SM
  const int want = zc_ceil_div(n_rows, 1024) > zc_ceil_div(n_req, 64) ? zc_ceil_div(n_rows, 1024) : zc_ceil_div(n_req, 64);
  const int grid = want > 296 ? 296 : want;
  return zc_cuda_status((int)zc_launch_early(k_page_tables, dim3(grid), dim3(kTabThreads), 0, (cudaStream_t)stream, log2,
                                             n_req, past, fresh, free_pages, n_free, free_state, table, table_width,
                                             kv_len, row_start, n_rows, slots, pos, free_out));
}

int zc_page_write(zc_pages* p, const void* k_rows, const void* v_rows, const int64_t row_strides[2],
                  const int32_t* slots, int n_rows, zc_stream_t stream) {
  if (!p || n_rows < 0 || !row_strides) return ZC_EINVAL;
  if (n_rows == 0) return ZC_OK;
  if (!k_rows || !v_rows || !slots) return ZC_EINVAL;
  if (!aligned16(k_rows) || !aligned16(v_rows) || !aligned4(slots)) return ZC_EALIGN;
  for (int i = 0; i < 2; ++i)
    if (row_strides[i] < 0 || row_strides[i] % 8) return ZC_EINVAL;
  const long long pieces = (long long)n_rows * p->cfg.n_kv_heads;
  const long long grid = (pieces + kUnroll * (kCopyThreads / 16) - 1) / (kUnroll * (kCopyThreads / 16));
  if (grid > 0x7fffffffLL) return ZC_EINVAL;
  const int64_t* s = p->cfg.strides;
  const cudaError_t e = zc_launch_early(
      k_page_write, dim3((int)grid), dim3(kCopyThreads), 0, (cudaStream_t)stream, p->k, p->v, 2 * s[0], 2 * s[1], 2 * s[2],
      p->page_log2, p->cfg.n_pages, p->cfg.n_kv_heads, (const char*)k_rows, (const char*)v_rows, 2 * row_strides[0],
      2 * row_strides[1], slots, pieces);
  p->launches += 1;
  return zc_cuda_status((int)e);
}

int zc_page_read(zc_pages* p, const int32_t* table, int table_width, int n_req, int l, void* K, void* V,
                 const int64_t kv_strides[3], zc_stream_t stream) {
  if (!p || !table || !K || !V || !kv_strides || table_width < 1 || n_req < 1 || l < 1) return ZC_EINVAL;
  if ((long long)l > (long long)table_width << p->page_log2) return ZC_ECAPACITY;
  if (!aligned16(K) || !aligned16(V) || !aligned4(table)) return ZC_EALIGN;
  for (int i = 0; i < 3; ++i)
    if (kv_strides[i] < 0 || kv_strides[i] % 8) return ZC_EINVAL;
  const int per_head = zc_ceil_div(l, kUnroll * (kCopyThreads / 16));
  const long long grid = (long long)per_head * n_req * p->cfg.n_kv_heads;
  if (grid > 0x7fffffffLL) return ZC_EINVAL;
  const int64_t* s = p->cfg.strides;
  const cudaError_t e = zc_launch_early(
      k_page_read, dim3((int)grid), dim3(kCopyThreads), 0, (cudaStream_t)stream, p->k, p->v, 2 * s[0], 2 * s[1], 2 * s[2],
      p->page_log2, p->cfg.n_pages, p->cfg.n_kv_heads, table, table_width, l, (char*)K, (char*)V, 2 * kv_strides[0],
      2 * kv_strides[1], 2 * kv_strides[2], per_head);
  p->launches += 1;
  return zc_cuda_status((int)e);
}

int zc_paged_attention(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table, int table_width,
                       const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows, int max_rows,
                       int window, int sinks, void* out, float* row_lse, void* workspace, size_t workspace_bytes,
                       zc_stream_t stream) {
  ZcPagedArgs a;
  const int rc = paged_args(p, q, q_strides, table, table_width, row_start, kv_len, n_req, n_rows, max_rows, window, sinks,
                            out, row_lse, workspace, &a);
  if (rc != ZC_OK || a.n_req == 0) return rc;
  const bool few = few_rows(a);
  if (workspace_bytes < (few ? zc_paged_decode_workspace() : zc_paged_chunk_workspace())) return ZC_ECAPACITY;
  if (!few && !zc_paged_chunk_fits(p->G, n_req, n_rows)) return ZC_ECAPACITY;
  const int e = few ? zc_launch_paged_decode(p, a, nullptr, (char*)workspace, (cudaStream_t)stream)
                    : zc_launch_paged_chunk(p, a, (char*)workspace, (cudaStream_t)stream);
  return zc_cuda_status(e);
}

int zc_scores_workspace(const zc_page_config* cfg, int max_rows, size_t* bytes) {
  const int rc = check_page_config(cfg);
  if (rc) return rc;
  if (max_rows < 0 || !bytes) return ZC_EINVAL;
  *bytes = logits_bytes(*cfg, max_rows);
  return ZC_OK;
}

int zc_paged_attention_scored(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table,
                              int table_width, const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows,
                              int max_rows, int window, int sinks, const int32_t* first, float* scores, void* out,
                              float* row_lse, void* workspace, size_t workspace_bytes, void* logits,
                              size_t logits_size, zc_stream_t stream) {
  ZcPagedArgs a;
  const int rc = paged_args(p, q, q_strides, table, table_width, row_start, kv_len, n_req, n_rows, max_rows, window, sinks,
                            out, row_lse, workspace, &a);
  if (rc != ZC_OK || a.n_req == 0) return rc;
  if (!scores || !row_lse) return ZC_EINVAL;
  if (!aligned16(scores) || !aligned4(first) || !aligned16(logits)) return ZC_EALIGN;
  const bool few = few_rows(a);
  if (few && !logits) return ZC_EINVAL;
  if (workspace_bytes < (few ? zc_paged_decode_workspace() : zc_paged_chunk_workspace())) return ZC_ECAPACITY;
  if (few ? logits_size < logits_bytes(p->cfg, a.max_rows) : !zc_paged_chunk_fits(p->G, n_req, n_rows)) return ZC_ECAPACITY;
  const cudaStream_t st = (cudaStream_t)stream;
  int e;
  if (few) {
    e = zc_launch_paged_decode(p, a, (float*)logits, (char*)workspace, st);
    if (e == cudaSuccess) e = zc_launch_score_add(p, a, (float*)logits, scores, first, nullptr, nullptr, 0, st);
  } else {
    e = zc_launch_paged_chunk(p, a, (char*)workspace, st);
    if (e == cudaSuccess) e = zc_launch_chunk_weights(p, a, scores, first, (char*)workspace, st);
  }
  return zc_cuda_status(e);
}

int zc_pages_shared_workspace(const zc_page_config* cfg, int n_req, int n_rows, size_t* workspace_bytes) {
  const int rc = zc_pages_workspace(cfg, n_req, n_rows, workspace_bytes);
  if (rc) return rc;
  *workspace_bytes = zc_paged_shared_workspace(*cfg, n_req, n_rows);
  return ZC_OK;
}

int zc_paged_attention_shared(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table,
                              int table_width, const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows,
                              int max_rows, const int32_t* group_start, const int32_t* shared_len, int n_groups,
                              float* scores, void* out, float* row_lse, void* workspace, size_t workspace_bytes,
                              void* logits, size_t logits_size, zc_stream_t stream) {
  ZcPagedArgs a;
  if (n_groups < 0 || (n_groups > 0 && (!group_start || !shared_len))) return ZC_EINVAL;
  const int rc = paged_args(p, q, q_strides, table, table_width, row_start, kv_len, n_req, n_rows, max_rows, 0, 0, out,
                            row_lse, workspace, &a);
  if (rc != ZC_OK || a.n_req == 0) return rc;
  if (!few_rows(a) || (long long)n_req * a.h_kv * ZC_PAGED_ROWS > 0x7fffffffLL) return ZC_EINVAL;
  if (scores && (!row_lse || !logits)) return ZC_EINVAL;
  if (!aligned4(group_start, shared_len) || !aligned16(scores) || !aligned16(logits)) return ZC_EALIGN;
  if (n_groups > ZC_PAGED_MAX_GROUPS || !zc_paged_chunk_fits(p->G, n_req, n_rows)) return ZC_ECAPACITY;
  if (workspace_bytes < zc_paged_shared_workspace(p->cfg, n_req, n_rows)) return ZC_ECAPACITY;
  if (scores && logits_size < logits_bytes(p->cfg, a.max_rows)) return ZC_ECAPACITY;
  const cudaStream_t st = (cudaStream_t)stream;
  float* kept = scores ? (float*)logits : nullptr;
  int e;
  // What sharing can save at most, by the table's width, against what its kernels take beside their keys: about 15 us, in
  // which 90 MB are read (8 requests behind 1000 tokens, 8 KV heads: 24 us shared, 14 as any).
  const int spare = n_req - (n_groups < n_req ? n_groups : n_req);
  const double saved = (double)spare * ((long long)table_width << p->page_log2) * p->cfg.n_kv_heads * (4.0 * ZC_D);
  if (n_groups > 0 && saved > 90e6) {
    e = zc_launch_paged_shared(p, a, group_start, shared_len, n_groups, kept, (char*)workspace, st);
  } else {
    e = zc_launch_paged_decode(p, a, kept, (char*)workspace, st);
  }
  if (scores && e == cudaSuccess)
    e = zc_launch_score_add(p, a, kept, scores, nullptr, group_start, shared_len, n_groups, st);
  return zc_cuda_status(e);
}

int zc_prefill_attention_window(zc_cache* c, const void* Q, const void* K, const void* V, int l,
                                const int64_t q_strides[3], const int64_t kv_strides[3], int window, int sinks,
                                void* O, float* row_lse, zc_stream_t stream) {
  if (!c || !Q || !K || !V || !O || !row_lse || !q_strides || !kv_strides) return ZC_EINVAL;
  if (l < 1 || window < 1 || sinks < 0) return ZC_EINVAL;
  if (l > c->cfg.max_prefill) return ZC_ECAPACITY;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(row_lse)) return ZC_EALIGN;
  for (int i = 0; i < 3; ++i)
    if (q_strides[i] < 0 || (q_strides[i] % 8) || kv_strides[i] < 0 || (kv_strides[i] % 8)) return ZC_EINVAL;
  if (q_strides[2] < ZC_D || kv_strides[2] < ZC_D) return ZC_EINVAL;
  return zc_cuda_status(zc_launch_prefill_window(c, Q, K, V, l, q_strides, kv_strides,
                                                 window > ZC_NO_WINDOW ? ZC_NO_WINDOW : window, sinks, O, row_lse,
                                                 (cudaStream_t)stream));
}

}  // extern "C"
