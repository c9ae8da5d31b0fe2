// Internal declarations of the full-precision pages: the host handle, what the attention kernels are
// given, and the arithmetic of visible keys that the kernels share.
#pragma once
#include <cuda.h>
#include <atomic>
#include <mutex>
#include "zc_internal.h"

#define ZC_PAGE_MAX_G 16            // most query heads per KV head
#define ZC_PAGED_ROWS 16            // rows (tokens x query heads of a KV head) the single-token kernel takes
#define ZC_PAGED_MAX_CTAS 160       // CTAs the workspace is sized for
#define ZC_NO_WINDOW (1 << 30)      // positions stay below it

// Several host threads may call with one handle.  The tensor maps are made by the first call that needs them.
struct zc_pages {
  zc_page_config cfg;
  char* k;
  char* v;
  int G, page_log2, n_sm;
  std::atomic<bool> maps_ready;
  std::mutex maps_guard;
  CUtensorMap k16, v16;    // boxes of 16 tokens x 128 elements (two 128-byte halves)
  CUtensorMap k64, v64;    // boxes of min(page, 64) tokens x 64 elements (x 2 halves from 64 on)
  std::atomic<long long> launches;
};

// One attention call, as the kernels see it.
struct ZcPagedArgs {
  const int32_t* table;
  const int32_t* row_start;
  const int32_t* kv_len;
  int table_width, n_req, n_rows, max_rows;
  int page_log2, n_pages;
  int h_q, h_kv, G;
  int window, sinks;       // window = ZC_NO_WINDOW: none
  const void* q;
  long long qs_row, qs_head;
  void* out;
  float* lse;              // may be null
};

// Keys that the rows at positions p_first .. p_last of a request may see, in blocks of 2^log2 keys:
// the first `nsb` blocks (sinks in front of the window), then blocks wb0, wb0 + 1, ... (the window).
// Position of virtual block vb: vb < nsb ? vb : wb0 + vb - nsb.
struct ZcSeen {
  int lo, hi;      // window part: keys lo .. hi - 1
  int sink_n;      // keys 0 .. sink_n - 1 lie in front of it and are seen as well
  int nsb, wb0, nb;
};
__device__ static inline ZcSeen zc_seen(int p_first, int p_last, int window, int sinks, int log2) {
  ZcSeen s;
  s.hi = p_last + 1 > 0 ? p_last + 1 : 0;
  const int lo = p_first - window + 1;
  s.lo = lo > 0 ? lo : 0;
  s.sink_n = sinks < s.lo ? sinks : s.lo;
  const int size = 1 << log2;
  s.nsb = (s.sink_n + size - 1) >> log2;
  s.wb0 = (s.lo >> log2) > s.nsb ? (s.lo >> log2) : s.nsb;
  const int end = (s.hi + size - 1) >> log2;
  s.nb = s.nsb + (end > s.wb0 ? end - s.wb0 : 0);
  return s;
}

// Workspace of one call: arrival counters, what the joining kernel is told, and the partial results that are joined.
size_t zc_paged_decode_workspace();
size_t zc_paged_chunk_workspace();
bool zc_paged_chunk_fits(int G, int n_req, int n_rows);   // the call's items fit the chunk kernel's shared memory
int zc_launch_paged_decode(zc_pages* p, const ZcPagedArgs& a, char* ws, cudaStream_t st);
int zc_launch_paged_chunk(zc_pages* p, const ZcPagedArgs& a, char* ws, cudaStream_t st);
int zc_launch_prefill_window(zc_cache* c, const void* Q, const void* K, const void* V, int l, const int64_t* qs,
                             const int64_t* ks, int window, int sinks, void* O, float* lse, cudaStream_t st);
int zc_paged_decode_error_code(int* out);
int zc_paged_chunk_error_code(int* out);
