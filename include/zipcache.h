/*
 * zipcache.h -- C ABI of the B200 (sm_100a) quantize-and-attend library.
 *
 * The library implements the mixed-precision KV-cache path of ZipCache:
 *   prefill:  probe attention (Eq. 9) -> normalised attention score (Eq. 8)
 *             -> split by saliency ratio (Alg. 2) -> channel-separable tokenwise
 *             quantisation (Alg. 1, Eq. 5, Eq. 6) -> packed 4-bit / 2-bit codes;
 *   decode:   append of the new token at full precision (Eq. 3, Alg. 3),
 *             single-query attention over the whole cache with in-kernel
 *             dequantisation (Eq. 4, Alg. 3), probe-row collection and the
 *             re-compression of every `window` generated tokens (Alg. 3).
 *
 * Conventions
 *   - "unit" = one (batch, KV head).  Query head h reads KV head h / G,
 *     G = n_q_heads / n_kv_heads.
 *   - Every pointer is tagged [host] or [device].  The library never allocates
 *     or frees device memory and never creates streams: the caller owns the
 *     cache buffer and the workspace, and all work is enqueued on the stream
 *     passed in.  Inputs may be released once the stream has passed the call.
 *   - Every function returns 0 (ZC_OK) or a negative status; nothing throws
 *     and device code never traps.  NaN / Inf in inputs give undefined values
 *     but no fault.
 *   - Device pointers must be 16-byte aligned (ZC_EALIGN otherwise).
 */
#ifndef ZIPCACHE_H_
#define ZIPCACHE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* zc_stream_t; /* a cudaStream_t */

enum { ZC_F16 = 0, ZC_BF16 = 1 };
/* How keys are quantised (values always by CSTQuant, Alg. 1).  ZC_K_CHANNEL is the paper's own
 * setting (Sec. 4.1, Table 1 last row, Alg. 2 "ChannelQuant"): Eq. 5 with minimum and maximum
 * taken over the tokens of a subset, one (s, z) pair per channel and none per token, which
 * saves 8 bytes per cached token. */
enum { ZC_K_CST = 0, ZC_K_CHANNEL = 1 };
/* Who shares a saliency decision (Sec. 4.2 speaks of the saliency "of each token"; the paper
 * does not say how heads are combined).  ZC_SCOPE_KV_HEAD: one decision per (batch row, KV head)
 * from that head's own normalised scores (Eq. 8 over its query heads).  ZC_SCOPE_TOKEN: one
 * decision per token of a batch row, shared by all its KV heads: the token's score is the mean
 * of its per-KV-head normalised scores, in the prompt and in every re-compressed window, so
 * every head of the row keeps the same tokens at the higher precision.  With ZC_SCOPE_TOKEN the
 * window is re-compressed by kernels of its own that follow the decode kernel of the call that
 * completes it (the heads' statistics must meet first), so it cannot be combined with
 * ZC_FLAG_OVERLAP_CALLS (zc_cache_bytes / zc_cache_init return ZC_EINVAL). */
enum { ZC_SCOPE_KV_HEAD = 0, ZC_SCOPE_TOKEN = 1 };

enum {
  ZC_OK = 0,
  ZC_EINVAL = -1,    /* bad shape / ratio / bit-width / stride / probe list */
  ZC_ECAPACITY = -2, /* more tokens than the cache or workspace was sized for */
  ZC_ESTATE = -3,    /* call out of order (e.g. decode before prefill) */
  ZC_EALIGN = -4,    /* pointer not 16-byte aligned */
  ZC_ECUDA = -5,     /* a CUDA runtime call or launch failed */
  ZC_ESCRATCH = -6   /* zc_decode_attention_noalloc: the call needs more scratch than the
                        library's built-in buffer holds */
};

#define ZC_MAX_WINDOW 128

/* zc_config.flags.  With ZC_FLAG_DEFER_APPEND, zc_append enqueues nothing: the new row is
 * taken straight from k_new / v_new by the next zc_decode_attention on the same cache and
 * stream, which also stores it into the tail (Alg. 3's concat and attention as one step: one
 * launch less and no wait between the two).  The caller then promises that k_new and v_new
 * stay valid and unchanged until the stream has passed that zc_decode_attention call.  Any
 * other call on the cache first performs the pending append as its own launch. */
#define ZC_FLAG_DEFER_APPEND 1
/* With ZC_FLAG_OVERLAP_CALLS the caller PROMISES that, on the stream it passes, a decode call of
 * this cache is preceded only by work that has completed or by other zc_decode_attention /
 * zc_append calls of this library (the layers of a benchmark, caches of independent requests),
 * with no kernel of another library between them.  The decode kernel then does not wait for the
 * kernel before it: consecutive calls run side by side on the GPU, ordered among themselves only
 * where their buffers require it (see zc_decode_attention), and a call is cut into few large
 * work items, which is best when several calls share the GPU.
 * Without the flag (the default) every decode kernel waits for everything that precedes it on
 * the stream before it reads q, k_new, v_new or the cache -- also when the kernel before it is
 * one that lets its successors start early (programmatic dependent launch), e.g. the projection
 * that produces q -- and a call is cut into items sized for a call that has the GPU to itself. */
#define ZC_FLAG_OVERLAP_CALLS 2
/* With ZC_FLAG_OUT_F32 zc_decode_attention stores its result as fp32 (out [device]
 * b x h_q x d floats) instead of rounding it to cfg.dtype.  A 16-bit output cannot be closer
 * to the exact result than half a unit in its last place (bf16: 2e-3 from |o| = 0.25 on), so
 * this is the form in which the kernel's own arithmetic (Eq. 4 over the dequantised cache)
 * can be compared with a reference at a tolerance below that. */
#define ZC_FLAG_OUT_F32 4
/* With ZC_FLAG_PARAMS_F16 the quantisation parameters are stored in 16 bits each, as Appendix A
 * counts them: the channel factors and the token scales as fp16 values, ROUNDED UP before the
 * codes are formed (a scale rounded down would no longer cover its token's range), the zero
 * points as 16-bit integers; a cached token then takes 8 bytes of parameters instead of 16.
 * For CSTQuant on keys and values (ZC_K_CST) at 2 or 4 bits; the window is re-compressed by
 * kernels of their own behind the decode kernel of the call that completes it, so the flag
 * cannot be combined with ZC_FLAG_OVERLAP_CALLS (ZC_EINVAL for either violation). */
#define ZC_FLAG_PARAMS_F16 8
/* With ZC_FLAG_GROUP_ALL_HEADS a token's scale and zero point are taken over the channels of ALL
 * KV heads of its batch row (Alg. 1 as printed: X in R^{l x hd}; Sec. 4.1 counts 2bl token
 * parameters per tensor), not over one head's head_dim channels; every head's tiles carry the
 * row's shared pair.  The heads must agree on the subsets, so it needs ZC_SCOPE_TOKEN (and with
 * it no ZC_FLAG_OVERLAP_CALLS); 16-bit classes are not admitted (ZC_EINVAL otherwise).
 * Channelwise keys have no token parameters: with ZC_K_CHANNEL only the values are grouped. */
#define ZC_FLAG_GROUP_ALL_HEADS 16

/* Plain-data configuration; set struct_size = sizeof(zc_config). */
typedef struct {
  int32_t struct_size;
  int32_t dtype;          /* ZC_F16 | ZC_BF16: type of Q, K, V, q, k, v, out */
  int32_t batch;          /* b */
  int32_t n_q_heads;      /* h_q, multiple of n_kv_heads, G <= 8 */
  int32_t n_kv_heads;     /* h_kv */
  int32_t head_dim;       /* d, must be 128 */
  int32_t max_prefill;    /* largest l accepted by zc_prefill_compress */
  int32_t max_new_tokens; /* decode capacity (tokens appended after prefill) */
  int32_t window;         /* tokens kept at full precision before re-compression
                             (Alg. 3 uses 100); 8 <= window <= ZC_MAX_WINDOW */
  int32_t bits_hi;        /* bit-width of salient tokens: 8, 4, 2, or 16 (kept as they are: the
                             "16/16" and "16/2" settings of Table 3) */
  int32_t bits_lo;        /* bit-width of regular tokens: 8, 4, 2 or 16; a cache with an 8-bit
                             class cannot also have a 16-bit one (ZC_EINVAL) */
  int32_t flags;          /* 0 or an OR of the ZC_FLAG_* values above */
  double saliency_ratio;  /* r in [0,1]; n_salient = floor(r * n) */
  int32_t k_scheme;       /* quantiser of the keys: ZC_K_CST (Alg. 1 on K and V) or ZC_K_CHANNEL
                             (channelwise keys, Sec. 4.1 last paragraph / Alg. 2; values stay CST) */
  int32_t scope;          /* ZC_SCOPE_KV_HEAD (0) or ZC_SCOPE_TOKEN: who shares a saliency decision */
} zc_config;

typedef struct zc_cache zc_cache; /* small host-side handle */

/* Sizes [host].  cache_bytes: device buffer for the compressed cache;
 * workspace_bytes: device scratch shared by all calls (in prefill: probe positions, probe-row
 * statistics and a dense copy of the probe rows; in decode: split-K partial results, with room
 * for 16 calls in flight together).  Either out pointer may be NULL. */
int zc_cache_bytes(const zc_config* cfg, size_t* cache_bytes, size_t* workspace_bytes);

/* Create a handle over caller-owned device memory `dev_mem` [device, >= cache_bytes,
 * 256-byte aligned].  No device work is enqueued.  *out is freed with zc_cache_free,
 * which releases the host handle only. */
int zc_cache_init(void* dev_mem, size_t bytes, const zc_config* cfg, zc_cache** out);
void zc_cache_free(zc_cache* c);

/* Probe selection (Sec. 4.3 "random+recent"): ascending positions made of the last
 * max(1, floor(rho_recent*l)) tokens plus floor(rho_random*l) of the others, drawn by a
 * partial Fisher-Yates shuffle driven by splitmix64(seed).  out [host] must hold
 * zc_probe_count(l, ...) entries; *n_out receives the count. */
int zc_probe_count(int l, double rho_recent, double rho_random);
int zc_default_probes(int l, double rho_recent, double rho_random, uint64_t seed,
                      int32_t* out, int* n_out);

/* Prefill compression (Alg. 2 without its attention-output line).
 *   Q [device] b x h_q x l x d, K, V [device] b x h_kv x l x d, element type cfg.dtype,
 *   d contiguous; q_strides / kv_strides [host] = strides of (batch, head, token) in
 *   ELEMENTS (multiples of 8).
 *   probe_pos [host] n_probe ascending token positions, the last one equal to l-1
 *   (Eq. 9's probe rows); ignored when salient_idx is given.
 *   salient_idx [device or NULL]: test hook -- b x h_kv x floor(r*l) ascending token
 *   indices to use as the salient set instead of computing Eq. 8 / the split.
 *   workspace [device] >= workspace_bytes from zc_cache_bytes.
 * Resets the cache to one compressed segment of l tokens and an empty tail. */
int zc_prefill_compress(zc_cache* c, const void* Q, const void* K, const void* V, int l,
                        const int64_t q_strides[3], const int64_t kv_strides[3],
                        const int32_t* probe_pos, int n_probe, const int32_t* salient_idx,
                        void* workspace, size_t workspace_bytes, zc_stream_t stream);

/* Prefill attention output (Eq. 2 with the causal mask; Alg. 2's line "O = FlashAttention(Q, K,
 * V)", Appendix B): O [device] b x h_q x l x d (contiguous, cfg.dtype) = Softmax(Q K^T /
 * sqrt(d)) V, row i over keys j <= i, and row_lse [device] b x h_q x l floats, every row's
 * base-2 log-sum-exp of its scaled logits (log2 sum_j 2^(q_i.k_j log2(e) / sqrt(d))).  Q, K, V and
 * their strides as for zc_prefill_compress.  The cache is not touched (the handle supplies the
 * shapes).  Needs the driver's tensor-map entry point (ZC_ECUDA "not supported" without it). */
int zc_prefill_attention(zc_cache* c, const void* Q, const void* K, const void* V, int l,
                         const int64_t q_strides[3], const int64_t kv_strides[3], void* O,
                         float* row_lse, zc_stream_t stream);

/* zc_prefill_compress for a caller that has just run zc_prefill_attention on the same Q and K:
 * row_lse [device] (that call's output) stands in for the first of the two probe-score passes
 * (Eq. 9's row statistics), which is then not run; everything else, and the resulting cache, is
 * the same. */
int zc_prefill_compress_lse(zc_cache* c, const void* Q, const void* K, const void* V, int l,
                            const int64_t q_strides[3], const int64_t kv_strides[3],
                            const int32_t* probe_pos, int n_probe, const float* row_lse,
                            void* workspace, size_t workspace_bytes, zc_stream_t stream);

/* Append (Eq. 3, Alg. 3): k_new, v_new [device] b x h_kv x d, contiguous, are copied
 * verbatim into the full-precision tail.  ZC_ECAPACITY beyond max_new_tokens.  With
 * ZC_FLAG_DEFER_APPEND the copy happens inside the next zc_decode_attention (see the flag). */
int zc_append(zc_cache* c, const void* k_new, const void* v_new, zc_stream_t stream);

/* Decode attention (Eq. 4, Alg. 3): q [device] b x h_q x d -> out [device] b x h_q x d,
 * softmax(q K^T / sqrt(d)) V over every cached token, codes dequantised in the kernel.
 * The step counter of the current window advances; on a probe step (is_probe_step != 0,
 * or one of the last five steps of a window) this step's attention over the tail's
 * tokens is added to the window statistics; the call that takes the window's last step
 * also re-compresses the tail into a new segment, inside the same kernel (no further launch,
 * no host synchronisation); with ZC_SCOPE_TOKEN or ZC_FLAG_PARAMS_F16 by five or six small kernels
 * launched behind it on the same stream (still no host synchronisation).
 * Only a call that follows a zc_append takes a step of Alg. 3; a further call on the same tail
 * (the same token queried again) attends the cache as it is and leaves the window's counters,
 * statistics and segments alone.
 * Ordering.  Default: the call's kernel starts its work after everything issued before it on
 * the stream has completed, whoever launched it.  With ZC_FLAG_OVERLAP_CALLS: consecutive calls
 * on one stream may run at the same time on the GPU; the library orders a call after the
 * earlier ones whenever it reads or overwrites one of their outputs, overwrites one of their
 * inputs, or updates the same cache's window statistics; it cannot see other aliasing, so q,
 * k_new, v_new and out of calls issued back to back must not overlap buffers that an earlier
 * call of the stream still uses in any other way, and (the flag's promise) no kernel of another
 * library may sit between the calls.  In both modes the workspace must not be used by calls on
 * another stream at the same time, and CUDA graphs captured from one stream must not be
 * replayed at the same time on several streams (the calls of a capture share one ordering
 * word per captured stream). */
int zc_decode_attention(zc_cache* c, const void* q, void* out, int is_probe_step,
                        void* workspace, size_t workspace_bytes, zc_stream_t stream);

/* ---- parity / export: canonical layouts written to caller buffers [device] ---- */
/* Normalised scores (Eq. 8) of the most recent compression: p_tilde b x h_kv x n floats,
 * n = l after prefill, window after a re-compression. */
int zc_export_scores(zc_cache* c, float* p_tilde, zc_stream_t stream);
/* Number of tokens in (segment, subset); subset 0 = salient, 1 = regular. */
int zc_segment_tokens(const zc_cache* c, int segment, int subset);
int zc_num_segments(const zc_cache* c);
int zc_tail_tokens(const zc_cache* c);
/* One subset of one segment, all units: idx b x h_kv x n int32 (ascending positions
 * within the segment); codes b x h_kv x n x (d*bits/8) bytes in canonical packing
 * (4-bit: element 2m low nibble, 2m+1 high nibble of byte m; 2-bit: element 4m+j in
 * bits [2j,2j+1] of byte m); sz b x h_kv x n x 2 floats (scale, zero point);
 * cf b x h_kv x d floats (channel factors).  tensor 0 = K, 1 = V.  Any out may be NULL.
 * A subset kept at 16 bits exports its rows' bytes as codes (256 per token) and nothing else.
 * Keys under ZC_K_CHANNEL have no per-token parameters and no channel factors: for tensor 0,
 * sz then receives b x h_kv x d x 2 floats, the (scale, zero point) of every channel, and cf
 * is left untouched. */
int zc_export_segment(zc_cache* c, int segment, int tensor, int subset, int32_t* idx,
                      uint8_t* codes, float* sz, float* cf, zc_stream_t stream);

/* Size of the scratch buffer built into the library for zc_decode_attention_noalloc. */
#define ZC_NOALLOC_SCRATCH_BYTES (4u << 20)

/* The paper has no counterpart for this entry point; it exists for integration reasons.
 * Same operation, arguments and state changes as zc_decode_attention, for callers that have
 * no way to hand the library a workspace: code that runs where device allocation is not
 * allowed or not possible -- a plug-in inside a serving process whose memory pool owns the
 * whole device and forbids further cudaMalloc calls, a latency-critical loop that must not
 * enter the allocator, a caller that has already given away its memory budget.  The split-K
 * partial results go to a fixed buffer of ZC_NOALLOC_SCRATCH_BYTES that is
 * part of the library image (every GPU that loads the library carries it until the process
 * ends); the caller still owns q [device] and out [device].  The call allocates and frees
 * nothing.
 *   - ZC_ESCRATCH, with nothing enqueued, when the cache's shape needs more than the
 *     built-in buffer (about batch * n_q_heads * (items + 8) * 528 bytes, items = split-K
 *     pieces per KV head, 8 = tiles of the full-precision tail; use zc_decode_attention with a
 *     caller workspace then).
 *   - The buffer's device address is looked up once per device (a synchronous runtime
 *     query), by zc_cache_init when a device is current there, else by the first call of
 *     this entry point on the device: that first call then belongs outside any stream capture.
 *   - All calls share the one buffer, whatever cache they work on.  Calls that follow one
 *     another in ONE stream get separate parts of it or are ordered by the library; calls in
 *     different streams, or from several host threads, that may run at the same time on the
 *     GPU overwrite each other's partial results.  Nothing in the buffer has to survive between calls and nothing in it
 *     has to be cleared: each call rewrites every word it later reads. */
int zc_decode_attention_noalloc(zc_cache* c, const void* q, void* out, int is_probe_step,
                                zc_stream_t stream);

/* ---- full-precision pages ------------------------------------------------------------------
 * Keys and values of requests whose prompts are not complete yet (or that are never compressed)
 * live at the input type in pages of `page_size` consecutive tokens of one request, all KV heads.
 * A request's pages are listed, in token order, in its row of a block table: table [device] n_req x
 * table_width int32, row-major; token t of request r is row t % page_size of page
 * table[r][t / page_size].  A slot is page * page_size + row.  The steps of a serving loop:
 * zc_page_tables (pages and slots for the step's new tokens), zc_page_write (their K / V rows into
 * the slots), zc_paged_attention (from the new tokens to everything cached), and, when a prompt is
 * complete, zc_page_read (its rows as the dense tensors zc_prefill_compress takes).
 * All lengths and tables are read on the device, so that a step can be captured in a CUDA graph
 * and replayed with other lengths of the same n_req / n_rows.  The calling thread's current device
 * must be the one that holds the buffers.
 * The kernels are launched while the stream's kernel before them still runs and wait for it before
 * they touch memory, so calls on one stream see each other's results as usual.  They are none of the
 * calls that ZC_FLAG_OVERLAP_CALLS lets a decode call overlap: let them complete before such a call. */
typedef struct {
  int32_t struct_size;    /* sizeof(zc_page_config) */
  int32_t dtype;          /* ZC_F16 | ZC_BF16 */
  int32_t n_q_heads;      /* h_q, multiple of n_kv_heads, at most 16 per KV head */
  int32_t n_kv_heads;     /* h_kv */
  int32_t head_dim;       /* must be 128 */
  int32_t page_size;      /* tokens per page: 16, 32, 64, 128 or 256 */
  int32_t n_pages;        /* n_pages * page_size <= 2^31 - 1 */
  int32_t reserved;       /* 0 */
  int64_t strides[3];     /* of (page, token, KV head) in ELEMENTS, for both tensors: multiples of 8,
                             at least 128 where the extent exceeds 1; d contiguous.  Any order of
                             the three is accepted. */
} zc_page_config;

typedef struct zc_pages zc_pages; /* small host-side handle; several host threads may use one at the same time (with
                                     workspaces and streams of their own), until zc_pages_free */

/* Device scratch [host] that zc_paged_attention needs for calls of up to n_req requests and n_rows rows
 * (partial results of rows whose keys several CTAs share; 43 MB for every admitted pair, since the CTAs and the rows
 * that each holds at once bound it: handles whose calls follow one another on a stream can share one, and
 * zc_page_write and zc_page_read need none).  ZC_ECAPACITY when one call cannot take so many:
 * n_req + n_rows / (2 * floor(128 / G)) may be 13000, G = n_q_heads / n_kv_heads.  Its first
 * ZC_PAGES_SYNC_BYTES must be zero before its first use (every call leaves them zero again); nothing else
 * in it needs initialisation or survives a call.  It must not be used by calls that may run at the same
 * time (other streams, graphs replayed side by side). */
#define ZC_PAGES_SYNC_BYTES 1024
int zc_pages_workspace(const zc_page_config* cfg, int n_req, int n_rows, size_t* workspace_bytes);
/* Handle over caller-owned pages K, V [device, 16-byte aligned].  No device work is enqueued. */
int zc_pages_init(void* k_pages, void* v_pages, const zc_page_config* cfg, zc_pages** out);
void zc_pages_free(zc_pages* p);

/* Block tables and slot maps of one step.  past, fresh [device] n_req int32: tokens request r has
 * cached, and tokens it adds now (negative values count as 0; sums must stay below 2^31).
 * free_pages [device] n_free int32: page ids; free_state [device] 3 int32: {next, end, -}: entries
 * next .. end - 1 of free_pages are free (end is taken as at most n_free).  Requests take pages in
 * their order: request r the next ceil((past + fresh) / page_size) - ceil(past / page_size) entries,
 * which are stored into its row of table behind those it holds.  Where the free list runs out, or
 * the table's row is full, a page is missing: its table entry (if the row has room) becomes -1.
 * Outputs [device], int32:
 *   table        in place, new entries only
 *   kv_len       n_req: past + fresh
 *   row_start    n_req + 1: prefix sums of fresh: the new tokens of request r are rows row_start[r]
 *                .. row_start[r + 1] - 1 of the step's row-wise tensors
 *   slots, pos   n_rows: slot and position of every row; slot -1 for a token whose page is missing;
 *                both -1 for rows behind the last request's (padding)
 *   free_out     3: {next + pages taken, end, pages missing}
 * No output may overlap past, fresh, free_pages or free_state (ZC_EINVAL): a step whose lengths feed the
 * next one's takes two sets of outputs in turn.
 * A step with pages missing must not be carried on with as it is: free pages and build it again. */
int zc_page_tables(int page_size, int n_req, const int32_t* past, const int32_t* fresh,
                   const int32_t* free_pages, int n_free, const int32_t* free_state, int32_t* table,
                   int table_width, int32_t* kv_len, int32_t* row_start, int n_rows, int32_t* slots,
                   int32_t* pos, int32_t* free_out, zc_stream_t stream);

/* New rows into pages: k_rows, v_rows [device] n_rows x h_kv x d of cfg.dtype, row_strides [host] =
 * strides of (row, head) in elements (multiples of 8), d contiguous; row i goes to slots[i] [device].
 * Rows whose slot is negative (or beyond the pages) are skipped.  Two rows with the same slot leave either's value
 * in each 16 bytes of it, head by head and in K and V apart: a mixture of both.  n_rows = 0 is a no-op. */
int zc_page_write(zc_pages* p, const void* k_rows, const void* v_rows, const int64_t row_strides[2],
                  const int32_t* slots, int n_rows, zc_stream_t stream);

/* Pages to dense tensors: the first l tokens of every request to K, V [device] n_req x h_kv x l x d,
 * kv_strides [host] = strides of (request, head, token) in elements, as zc_prefill_compress takes
 * them.  Tokens on pages outside [0, n_pages) come as zeros. */
int zc_page_read(zc_pages* p, const int32_t* table, int table_width, int n_req, int l, void* K, void* V,
                 const int64_t kv_strides[3], zc_stream_t stream);

/* Attention from each request's newest tokens to its cached ones (Eq. 2 and Eq. 4 over pages): the
 * rows row_start[r] .. row_start[r + 1] - 1 of q are the last n_r of the request's kv_len[r] tokens,
 * whose K / V rows are in the pages already; row i of them, at position p = kv_len[r] - n_r + i, sees
 * the keys j <= p and, with window > 0, of those only j > p - window and the first `sinks` tokens
 * (j < sinks).  window = 0: no window.
 *   q [device] n_rows x h_q x d, q_strides [host] = strides of (row, head) in elements (multiples of
 *   8); table [device] n_req x table_width; row_start [device] n_req + 1 ascending; kv_len [device]
 *   n_req; out [device] n_rows x h_q x d, contiguous, cfg.dtype; row_lse [device or NULL] n_rows x h_q
 *   floats, base-2 log-sum-exp of the scaled logits (as zc_prefill_attention's).
 *   max_rows [host]: a bound on n_r that the caller vouches for; it chooses the kernel, and rows of
 *   a request beyond it may be left as they were.
 * A row that sees no key (kv_len[r] < n_r) gives 0 and a log-sum-exp of -inf.  Rows of out outside
 * row_start[0] .. row_start[n_req] - 1 are left as they were.  Slots that no row of a request sees are
 * not read into its results, whatever they hold: pages that lie wholly outside the window and the sinks
 * may have been given away (any table entry).  kv_len beyond the table's width is taken as the width's
 * tokens.  Keys on pages outside [0, n_pages) give undefined values, no fault. */
int zc_paged_attention(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table,
                       int table_width, const int32_t* row_start, const int32_t* kv_len, int n_req,
                       int n_rows, int max_rows, int window, int sinks, void* out, float* row_lse,
                       void* workspace, size_t workspace_bytes, zc_stream_t stream);

/* zc_paged_attention for requests that begin alike: n_groups groups of consecutive requests, group g the requests
 * group_start[g] .. group_start[g + 1] - 1, the first shared_len[g] tokens of which are the same ones (a system prompt, a
 * document): their tables list the same pages for them, or copies of the same rows where a page is not filled by them.
 * Those keys and values are read once for all rows of the group, through the table of the first of its requests that has
 * rows in the call, instead of once per request (tables of requests without rows may hold anything).
 * group_start [device] n_groups + 1 ascending, shared_len [device] n_groups; requests in no group, and groups too short to
 * be worth it (down to groups of one), are attended like any.  At most 1024 groups (ZC_ECAPACITY).
 * Of a group's shared tokens those count that lie before every new row of its requests.
 *   max_rows * G must be at most 16 (ZC_EINVAL): generated tokens, one or a few per request; a chunk reads each
 *   key once for 128 / G of its tokens as it is, and is zc_paged_attention's.
 *   scores [device or NULL]: as zc_paged_attention_scored, with shared_len in place of first (0 for requests in no
 *   group), and logits likewise.
 *   workspace: of zc_pages_shared_workspace for the call's n_req and n_rows (or more), zeroed in front as zc_pages_workspace
 *   says, whose calls it serves as well.
 * Results are zc_paged_attention's up to rounding: keys are added up in another order, and the weights of keys that are
 * read once for a group are rounded to the input type (by 2^-8 of them at most in bf16, 2^-11 in fp16), as a chunk's are,
 * where zc_paged_attention holds those of so few rows in two parts.  So an output is off by as much of the weighted mean of
 * |v| more, in calls and groups that are large enough to be worth it (by the table's width, the lengths and the number of
 * requests), and in none that is attended like any. */
int zc_paged_attention_shared(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table,
                              int table_width, const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows,
                              int max_rows, const int32_t* group_start, const int32_t* shared_len, int n_groups,
                              float* scores, void* out, float* row_lse, void* workspace, size_t workspace_bytes,
                              void* logits, size_t logits_bytes, zc_stream_t stream);
int zc_pages_shared_workspace(const zc_page_config* cfg, int n_req, int n_rows, size_t* workspace_bytes);

/* ---- thinning out ---------------------------------------------------------------------------
 * A request that may not grow keeps the tokens that attention has used.  zc_paged_attention_scored adds up every
 * cached token's weight, zc_page_select lists, per KV head, the tokens to keep by it, zc_page_compact moves their rows
 * to the front of the request's pages and gives the pages behind them back.  Afterwards the request has kept_len tokens
 * in its old order, and goes on as any other (its next token's position in the text is the caller's to know). */

/* zc_paged_attention that also adds up the weights of the cached tokens: for token j of request r and KV head h
 *   A[j, h] = sum over the request's rows i that see j, and the query heads of h, of 2^(s_ij - row_lse_i),
 * s the scaled logits (base 2).  Tokens that came with this call (the last n_r of kv_len[r]) start from A, older ones
 * add it to the score they have; so a slot needs no clearing before a new token takes it.
 *   scores [device, 16-byte aligned] n_pages x h_kv x page_size floats, contiguous, indexed by slot as the pages are;
 *   first [device or NULL] n_req: tokens before first[r] have no score (pages that other requests of the call share, say),
 *   theirs are left as they were, as are those of tokens that no row of the call sees.  A slot that two requests of the
 *   call score ends with a number that is neither's sum, nor the same every time: the logits that single tokens leave are
 *   one place to a slot.  It lies between 0 and the old score plus either's rows times G; other slots are not touched by it.
 *   row_lse must be given.  Sums are fp32, of fp32 weights, in a fixed order.  A row with a logit that is NaN or +inf (or
 *   with none above -inf) has no weights: the tokens that it sees get NaN.
 *   logits [device, 16-byte aligned]: scratch of calls whose max_rows * G is at most 16 (zc_scores_workspace for that
 *   max_rows; none for others, NULL then).  Nothing in it survives a call; it must not be used by calls that may run at
 *   the same time.
 * Everything else as zc_paged_attention, whose outputs it gives bit for bit. */
int zc_paged_attention_scored(zc_pages* p, const void* q, const int64_t q_strides[2], const int32_t* table,
                              int table_width, const int32_t* row_start, const int32_t* kv_len, int n_req, int n_rows,
                              int max_rows, int window, int sinks, const int32_t* first, float* scores, void* out,
                              float* row_lse, void* workspace, size_t workspace_bytes, void* logits,
                              size_t logits_bytes, zc_stream_t stream);
/* Bytes [host] of the logits' scratch: 4 per slot, query head and row. */
int zc_scores_workspace(const zc_page_config* cfg, int max_rows, size_t* bytes);

/* Which tokens a request keeps, per KV head: the first first[r] ones (NULL: 0), the last `recent` ones, and of those
 * between the ones with the highest scores, as many as make keep[r] tokens in all (at most max_keep; equal scores: the
 * lower position; a NaN is below every number).  keep, first [device] n_req; negative values count as 0.
 *   scores as zc_paged_attention_scored leaves them (16-byte aligned);
 *   kept [device] n_req x h_kv x max_keep int32: positions, ascending, -1 behind them;  kept_len [device] n_req: how
 *   many, the same for all heads.
 * first[r] + recent tokens are kept even where keep[r] is less.  A request that has no more than its keep[r] (even where
 * that is more than max_keep), or whose first and recent tokens alone are more than max_keep, stays as it is:
 * kept_len[r] = kv_len[r] (of which kept lists max_keep at most).  Outputs may not overlap inputs. */
int zc_page_select(zc_pages* p, const int32_t* table, int table_width, const int32_t* kv_len, int n_req,
                   const float* scores, const int32_t* keep, int recent, const int32_t* first, int32_t* kept,
                   int max_keep, int32_t* kept_len, zc_stream_t stream);

/* Moves, in K, V and (unless NULL) scores, the rows of the kept tokens to the first kept_len[r] slots of their request,
 * head by head, in place: token i of KV head h is then the one that was token kept[r][h][i].  kept [device] n_req x h_kv
 * x max_keep, the first kept_len[r] of each ascending in [0, kv_len[r]) (zc_page_select's, or a list of the caller's;
 * others give undefined rows of that request, no fault); requests with kept_len[r] >= kv_len[r], or above max_keep, are
 * left alone.  What lies behind the kept tokens is left as it is.  All pages of a request's kv_len[r] tokens must be
 * its own, but those whose tokens all stay where they are (pages of a shared beginning that first[r] covers).
 * The pages behind the kept tokens, request by request, are put back in front of the free ones, where zc_page_tables
 * took them from: free_pages [device] n_free, free_state, free_out [device] 3 as there: free_out = {next - pages, end,
 * pages that found no room in front of next: 0 where all came from this list}.  Entries outside [0, n_pages) are no pages
 * (a step that ran out of them leaves such) and are not put back.  All three NULL: none.  n_req = 0 is a no-op: free_out is
 * not written.  The table is left as it is; its entries behind the kept tokens' pages mean nothing any more.  Outputs may
 * not overlap inputs. */
int zc_page_compact(zc_pages* p, const int32_t* table, int table_width, const int32_t* kv_len, int n_req,
                    const int32_t* kept, int max_keep, const int32_t* kept_len, float* scores, int32_t* free_pages,
                    int n_free, const int32_t* free_state, int32_t* free_out, zc_stream_t stream);

/* zc_prefill_attention with a sliding window: row i sees the keys j <= i with j > i - window, and the
 * first `sinks` tokens (j < sinks); window >= 1, sinks >= 0.  Arguments, outputs and errors as there.
 * row_lse belongs to the windowed rows: zc_prefill_compress_lse wants zc_prefill_attention's, and decode attention over
 * a compressed cache knows no window. */
int zc_prefill_attention_window(zc_cache* c, const void* Q, const void* K, const void* V, int l,
                                const int64_t q_strides[3], const int64_t kv_strides[3], int window,
                                int sinks, void* O, float* row_lse, zc_stream_t stream);

/* Kernel launches enqueued through this handle since it was created. */
int64_t zc_pages_launch_count(const zc_pages* p);

/* Algorithmic bytes one zc_decode_attention call must read in the cache's current
 * state (packed codes + per-token parameters + tail + channel factors + q and out). */
int64_t zc_decode_bytes(const zc_cache* c);
/* Kernel launches enqueued by this library since the handle was created. */
int64_t zc_launch_count(const zc_cache* c);

/* Synchronises the device and reads the library's device-side error word into *code
 * [host]: 0 = none, 1 = a bounded wait on an asynchronous copy inside the decode kernel
 * ran out, 2 = a bounded wait for an earlier decode call of the stream ran out, 3 = a bounded wait
 * on the tensor cores inside a probe-score or prefill-attention kernel ran out, 4 = a bounded wait inside a paged-attention or windowed prefill-attention kernel ran out (outputs are then invalid).  Device code never traps or spins forever. */
int zc_device_status(int* code);

/* Host-only model of the ordering the library applies to zc_decode_attention calls issued on
 * one stream (the contract stated at zc_decode_attention): what each call's kernel waits for
 * before it reads its inputs and before it writes.  These two functions make no CUDA call,
 * need no device and keep a table of their own, apart from the one real calls use; they exist
 * so that the rules can be checked on any machine.  Not thread-safe.
 *
 * zc_order_model_reset forgets every stream and cache of the model.
 *
 * zc_order_model_call books one call.  stream_id: any integer naming the stream; cache_id in
 * [0, 16) names the cache; addr [host] = the addresses of q, k_new, v_new, out as integers
 * (k_new = v_new = 0: the call changes nothing in the cache), of io_bytes (q, out) and kv_bytes (k_new,
 * v_new); collect = is_probe_step; ws_addr / ws_bytes = the workspace, need = the bytes one
 * call uses of it; capture_id = 0 outside stream capture, else the capture's id.
 * result [host, 8 ints] = {epoch_start (1: launched without early start, everything issued
 * before it on the stream has completed), e (index of the call in its epoch), need_start
 * (the first need_start calls of the epoch have completed before this one reads its inputs;
 * <= 0: none), need_end (likewise before it writes anything), slot (workspace region and
 * arrival counter), tag (12-bit epoch number), record (stream record used), drain (1: the
 * record was taken from another stream, which a real call drains first)}.
 * Returns ZC_OK, or ZC_EINVAL (null pointer, cache_id out of range, need = 0 or > ws_bytes).
 */
void zc_order_model_reset(void);
int zc_order_model_call(uint64_t stream_id, int cache_id, const uint64_t addr[4], uint64_t io_bytes,
                        uint64_t kv_bytes, int collect, uint64_t ws_addr, uint64_t ws_bytes,
                        uint64_t need, uint64_t capture_id, int result[8]);

const char* zc_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* ZIPCACHE_H_ */
