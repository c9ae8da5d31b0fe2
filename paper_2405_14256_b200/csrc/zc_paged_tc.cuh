// What the kernels of the paged path share that work on chunks with tcgen05: a request's rows, tiles of query rows
// (token * G + head, 128 / G tokens to a tile) and their tensor map, paired arithmetic, and small warp helpers.
#pragma once
#include "zc_paged.cuh"

namespace {

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
// Q rows of one tile half: 64 channels x G heads x tokens, from (channel half kb, head, token) of batch row b on.
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
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 d, a, b;\n"
      " mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// The loads that wrote v[0 .. 31] have completed (the operands keep their uses behind the wait).
__device__ __forceinline__ void tmem_wait32(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                 "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
// One thread of the (converged) warp, the same each time.  What it issues is computed by the whole warp
// from values that are the same in all lanes: the operands of tcgen05.mma then live in uniform registers
// instead of being moved there one by one (75 against 48 cycles from one 128 x 64 x 16 product to the next).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
inline int tokens_per_tile(int G) { return kM / G; }
// Q as (channels, query heads, tokens, batch rows), boxes of 64 channels x G heads x tpt tokens.
inline bool make_q_map(CUtensorMap* map, const void* q, int dtype, int h_q, int G, long long tokens, int batch,
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

}  // namespace
