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
static_assert(ZC_PAGED_MAX_CTAS * 4 + 12 <= ZC_PAGES_SYNC_BYTES, "a counter per CTA, two of the weights' kernel, ZcGroups::told");
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
  CUtensorMap k128;        // boxes of min(page, 128) tokens x 64 elements
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

// Groups of requests with the same first keys, as the kernels of the shared and of the own keys and the joining one see them.
#define ZC_PAGED_MAX_GROUPS 1024
#define ZC_CHUNK_PART_ROWS 256                                   // a piece of the chunk kernel: [channels / 4][row] float4,
#define ZC_CHUNK_PART_BYTES (ZC_CHUNK_PART_ROWS * (128 * 4 + 8))   // then (maximum, sum) [row]
struct ZcGroups {
  const int32_t* start;    // [n + 1] the groups' requests
  const int32_t* shared;   // [n] tokens that a group's tables begin with alike
  int n, most;             // groups; items of a KV head that there is room for
  // the shared keys' kernel
  int* told;               // 1 + the CTAs that work on them, once one of them knows; zero before and after every call
  int* head;               // how many these are
  int* keys;               // [n] how many of the shared tokens the call reads once
  int* lead;               // [n] the request through whose table: the group's first that has rows (others may be anything)
  int4* info;              // [request] (its group's keys, its first row among the group's, the group's first item, -)
  int* cut;                // [item][KV head] 0: the result is with the rows; c: in pieces, the second CTA c's
  int* last;               // [CTA] the last of the CTAs that have pieces of the item that the border before this one cuts
  const int* used;         // [CTA] its share is not empty
  const char* parts;       // [CTA][2] pieces
  float* rows;             // (maximum, sum, -, -, 128 sums) of each (row, query head)
  // the own keys' kernel
  int4* own;               // [request] (where its blocks begin on a KV head's line: low and high word, its group's keys,
                           // its length on the line)
  long long* own_line;     // a KV head's line, a warp's stretch of all of them
  float* own_rows;         // (maximum, sum, -, -, 128 sums) of each row of each piece
};

// Workspace of one call: arrival counters, what the joining kernel is told, and the partial results that are joined.
size_t zc_paged_decode_workspace();
size_t zc_paged_chunk_workspace();
bool zc_paged_chunk_fits(int G, int n_req, int n_rows);   // the call's items fit the chunk kernel's shared memory
// logits: where they are kept, [page][KV head][token][max_rows * G], scaled, base 2; or null.
int zc_launch_paged_decode(zc_pages* p, const ZcPagedArgs& a, float* logits, char* ws, cudaStream_t st);
int zc_launch_paged_chunk(zc_pages* p, const ZcPagedArgs& a, char* ws, cudaStream_t st);
size_t zc_paged_shared_workspace(const zc_page_config& c, int n_req, int n_rows);
int zc_launch_paged_shared(zc_pages* p, const ZcPagedArgs& a, const int32_t* group_start, const int32_t* shared_len,
                           int n_groups, float* logits, char* ws, cudaStream_t st);
// go: false only asks for the shared memory that the launch needs.
int zc_launch_own_keys(zc_pages* p, const ZcPagedArgs& a, const ZcGroups& gr, int tpt, float* logits, bool go, cudaStream_t st);
// group_start, shared_len, n_groups: tokens before a group's shared_len have no score; else first (may be null) says so.
int zc_launch_score_add(zc_pages* p, const ZcPagedArgs& a, const float* logits, float* scores, const int32_t* first,
                        const int32_t* group_start, const int32_t* shared_len, int n_groups, cudaStream_t st);
int zc_launch_chunk_weights(zc_pages* p, const ZcPagedArgs& a, float* scores, const int32_t* first, char* ws, cudaStream_t st);
int zc_launch_prefill_window(zc_cache* c, const void* Q, const void* K, const void* V, int l, const int64_t* qs,
                             const int64_t* ks, int window, int sinks, void* O, float* lse, cudaStream_t st);
int zc_paged_decode_error_code(int* out);
int zc_paged_chunk_error_code(int* out);
int zc_paged_weights_error_code(int* out);
int zc_paged_own_error_code(int* out);
