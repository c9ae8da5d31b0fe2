// Attention of a few query rows (at most 8 or 16) over one block of 16 keys and values in shared memory, by one warp: what
// the kernels of single tokens share.  The query rows are the N dimension of the tensor-core tiles.
#pragma once
#include "zc_layout.cuh"
#include "zc_paged_tc.cuh"

namespace {

constexpr int kBlkLog2 = 4, kBlk = 1 << kBlkLog2;      // keys of a block
constexpr int kHalf = kBlk * ZC_D * 2;                 // 4 KB: keys (or values) of a block, [2][16][128 B]
constexpr float kTau = 8.f;

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

// Rows row = oct + 8 nt of a unit as B fragments, two consecutive channels a register.
template <typename T, int NT>
__device__ __forceinline__ void load_rows(const ZcPagedArgs& a, int row0, int kv, int rows, uint32_t (&qf)[NT][8][2]) {
  const int lane = threadIdx.x & 31, quad = lane & 3, oct = lane >> 2;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = oct + 8 * nt, tok = row / a.G;
    const T* qp = reinterpret_cast<const T*>(a.q) + (long long)(row0 + tok) * a.qs_row +
                  (long long)(kv * a.G + (row - tok * a.G)) * a.qs_head + 2 * quad;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      qf[nt][ks][0] = row < rows ? *reinterpret_cast<const uint32_t*>(qp + 16 * ks) : 0u;
      qf[nt][ks][1] = row < rows ? *reinterpret_cast<const uint32_t*>(qp + 16 * ks + 8) : 0u;
    }
  }
}
// Positions of this thread's rows (rows 2 quad, 2 quad + 1 of each group of 8), the first at p0; -1 beyond the rows.
template <int NT> __device__ __forceinline__ void row_positions(const ZcPagedArgs& a, int p0, int rows, int (&pos)[NT][2]) {
  const int quad = threadIdx.x & 3;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 8 * nt + 2 * quad + e;
      pos[nt][e] = row < rows ? p0 + row / a.G : -1;
    }
}
// Where the logits of key0 and its rows are kept: [page][KV head][token][max_rows * G].
__device__ __forceinline__ float* logits_of(float* logits, const ZcPagedArgs& a, int page, int kv, int key0) {
  return logits + ((((long long)page * a.h_kv + kv) << a.page_log2) + (key0 & ((1 << a.page_log2) - 1))) * (a.max_rows * a.G);
}

// What a warp has of its rows: channels 16 i + oct (+ 8) of rows 2 quad, 2 quad + 1 of each group of 8, before the
// division by the sums, which are this thread's own (of keys oct, oct + 8 of every block).
template <int NT> struct RowState {
  float o[NT][8][4], m[NT][2], s[NT][2], raw[NT][2];   // raw: q.k of the maximum
  bool far;                                            // a row of the warp has its maximum beyond kFarMax
  __device__ __forceinline__ void clear() {
    far = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
      m[nt][0] = m[nt][1] = kNoMax;
      raw[nt][0] = raw[nt][1] = 0.f;
      s[nt][0] = s[nt][1] = 0.f;
    }
  }
};

// The block of keys from key0 on, keys at shared address kt, values at vt (`values` as a pointer); logits: where its logits
// are kept (WEIGHTS; null: nowhere).
template <typename T, int NT, bool WEIGHTS>
__device__ __forceinline__ void attend_block(RowState<NT>& x, const uint32_t (&qf)[NT][8][2], const int (&pos)[NT][2],
                                             uint32_t kt, uint32_t vt, char* values, int key0, int p_first, int p_last,
                                             const ZcSeen& seen, const ZcPagedArgs& a, int rows, float* logits) {
  const int lane = threadIdx.x & 31, quad = lane & 3, oct = lane >> 2;
  const float scale = kLog2e * rsqrtf((float)ZC_D);
  // ---- S^T = K Q^T ----
  float sc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[nt][e] = 0.f;
  const int lrow = lane & 15;                         // matrices 0, 2: keys 0-7; 1, 3: keys 8-15
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) {
    const int chunk = 2 * ks + (lane >> 4);
    uint32_t kf[4];
    ldmatrix_x4(kf, kt + (chunk >> 3) * (kBlk * 128) + lrow * 128 + (((chunk & 7) ^ (lrow & 7)) << 4));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) zc_mma16816<T>(sc[nt], kf, qf[nt][ks][0], qf[nt][ks][1]);
  }
  // ---- masks: only blocks at a border ----
  if (key0 + kBlk - 1 > p_first || (key0 <= p_last - a.window && key0 + kBlk > a.sinks)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = key0 + oct + 8 * (e >> 1), p = pos[nt][e & 1];
        const bool on = key <= p && (key > p - a.window || key < a.sinks);
        if (!on) sc[nt][e] = -INFINITY;
      }
    // values that no row sees may hold anything (2^-inf = 0 times NaN is NaN): zeros in their place
    const int vr = lane >> 1, vkey = key0 + vr;
    const bool dead = vkey >= seen.hi || (vkey < seen.lo && vkey >= seen.sink_n);
    if (dead) {
      char* at = values + (lane & 1) * (kBlk * 128) + vr * 128;
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(at + 16 * i) = make_uint4(0, 0, 0, 0);
    }
    async_proxy_fence();   // the stage's next copy is ordered behind these stores
    __syncwarp();
  }
  // ---- the logits, for the keys' weights: [page][KV head][token][row] ----
  if (WEIGHTS && logits) {
    const int per = a.max_rows * a.G;
    float* at = logits + oct * per;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = 8 * nt + 2 * quad + (e & 1);
        if (row < rows) at[(e >> 1) * 8 * per + row] = sc[nt][e] * scale;
      }
  }
  // ---- running maximum and sum ----
  uint32_t pf[NT][2], rest[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float mx[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      mx[e] = fmaxf(sc[nt][e], sc[nt][e + 2]);
#pragma unroll
      for (int i = 4; i < 32; i <<= 1) mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], i));
    }
    const float top[2] = {mx[0], mx[1]};
    mx[0] *= scale;
    mx[1] *= scale;
    const bool grow0 = mx[0] > x.m[nt][0] + kTau, grow1 = mx[1] > x.m[nt][1] + kTau;
    if (__any_sync(0xffffffffu, grow0 || grow1)) {
      const float al0 = grow0 ? zc_exp2(x.m[nt][0] - mx[0]) : 1.f, al1 = grow1 ? zc_exp2(x.m[nt][1] - mx[1]) : 1.f;
      if (grow0) x.m[nt][0] = mx[0];
      if (grow1) x.m[nt][1] = mx[1];
      if (grow0) x.raw[nt][0] = top[0];
      if (grow1) x.raw[nt][1] = top[1];
      x.far = x.far || __any_sync(0xffffffffu, !(fmaxf(grow0 ? fabsf(mx[0]) : 0.f, grow1 ? fabsf(mx[1]) : 0.f) < kFarMax));
      x.s[nt][0] *= al0;
      x.s[nt][1] *= al1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x.o[nt][i][0] *= al0;
        x.o[nt][i][1] *= al1;
        x.o[nt][i][2] *= al0;
        x.o[nt][i][3] *= al1;
      }
    }
    float less[2] = {x.m[nt][0], x.m[nt][1]};
    if (x.far) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[nt][e] -= x.raw[nt][e & 1];
      less[0] = less[1] = 0.f;
    }
    const float p0 = zc_exp2(fmaf(sc[nt][0], scale, -less[0])), p1 = zc_exp2(fmaf(sc[nt][1], scale, -less[1]));
    const float p2 = zc_exp2(fmaf(sc[nt][2], scale, -less[0])), p3 = zc_exp2(fmaf(sc[nt][3], scale, -less[1]));
    x.s[nt][0] += p0 + p2;
    x.s[nt][1] += p1 + p3;
    const uint32_t w0 = pack2<T>(p0, p1), w1 = pack2<T>(p2, p3);   // keys 0-7 of the block, keys 8-15
    const float2 h0 = unpack2<T>(w0), h1 = unpack2<T>(w1);
    pf[nt][0] = movmatrix_trans(w0);
    pf[nt][1] = movmatrix_trans(w1);
    rest[nt][0] = movmatrix_trans(pack2<T>(p0 - h0.x, p1 - h0.y));
    rest[nt][1] = movmatrix_trans(pack2<T>(p2 - h1.x, p3 - h1.y));
  }
  // ---- O^T += V^T P^T ----
  const int vrow = (lane & 7) + ((lane >> 4) << 3);   // matrices 0, 1: keys 0-7; 2, 3: keys 8-15
#pragma unroll
  for (int m2 = 0; m2 < 8; m2 += 2) {   // two tiles of channels at a time, so that no product waits for the one before
    uint32_t vf[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int chunk = 2 * (m2 + u) + ((lane >> 3) & 1);
      ldmatrix_x4_trans(vf[u], vt + (chunk >> 3) * (kBlk * 128) + vrow * 128 + (((chunk & 7) ^ (vrow & 7)) << 4));
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < 2; ++u) zc_mma16816<T>(x.o[nt][m2 + u], vf[u], pf[nt][0], pf[nt][1]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < 2; ++u) zc_mma16816<T>(x.o[nt][m2 + u], vf[u], rest[nt][0], rest[nt][1]);
  }
}

}  // namespace
