// What the paged kernels share: bounded waits of a warp, tensor-map copies of page rows, output rows, tensor maps, and
// launches that may start beside the kernel they follow.
#pragma once
#include <cfloat>
#include "zc_pages.h"
#include "zc_tc.cuh"

bool zc_page_maps(zc_pages* p);   // encodes the handle's tensor maps (once); false: not supported

namespace {

// The two values that pack2 rounded, as they are held.
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

// a * b / c; the quotient of 32-bit numbers where they fit (a <= ZC_PAGED_MAX_CTAS).
static_assert(ZC_PAGED_MAX_CTAS < 256, "a * b < 2^32");
__device__ __forceinline__ long long zc_muldiv(int a, long long b, int c) {
  return b < (1 << 24) ? (long long)((uint32_t)a * (uint32_t)b / (uint32_t)c) : a * b / c;
}

constexpr float kNoMax = -FLT_MAX;                     // running maximum before any key
// The weights' exponents are (q.k) * scale - m, m the scaled maximum rounded to fp32: off by 2^-24 of m, for all of a row's keys
// alike, which cancels up to here (a shift of 4 at most).  Beyond, the maximum's own q.k is taken off before the scaling.
constexpr float kFarMax = 67108864.f;

// bar_wait of a whole warp, with one answer for all lanes: a lane whose wait ran out must not part from the others.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity));
}
// Before a warp leaves: what it asked for has arrived (or the bound has run out once more).
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) { (void)bar_wait(bar, parity); }

// One box of a page: rows `row` ... of it, half `half` of the channels on.
__device__ __forceinline__ void page_copy(const CUtensorMap* map, uint32_t dst, uint64_t* bar, int row, int half,
                                          int head, int page) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], "
      "[%7];\n" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(half), "r"(head), "r"(page), "r"(zc_smem_u32(bar))
      : "memory");
}

// Output row `at` (128 channels, a warp holds four each) from sum = sum of the weights 2^(s - m) and
// acc = sum of the weighted values; a row without keys (sum 0) gives 0 and a log-sum-exp of -inf.
template <typename T>
__device__ __forceinline__ void store_row(void* out, float* lse, long long at, int lane, float m, float sum, float4 acc) {
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  const uint2 w = make_uint2(pack2<T>(acc.x * inv, acc.y * inv), pack2<T>(acc.z * inv, acc.w * inv));
  *reinterpret_cast<uint2*>(reinterpret_cast<T*>(out) + at * ZC_D + 4 * lane) = w;
  if (lse && lane == 0) lse[at] = sum > 0.f ? m + log2f(sum) : -INFINITY;
}

// Tensor map in the 128-byte swizzle; strides in bytes.  False when the driver's entry point is missing
// or refuses the tensor.
inline bool zc_encode_map(CUtensorMap* map, int dtype, int rank, const void* at, const cuuint64_t* dims,
                          const cuuint64_t* strides, const cuuint32_t* box) {
  typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                               const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                               CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static EncodeFn encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      return (EncodeFn)f;
    cudaGetLastError();
    return (EncodeFn) nullptr;
  }();
  if (!encode) return false;
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return encode(map, dtype == ZC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                (cuuint32_t)rank, const_cast<void*>(at), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The opt-in to large shared memory, once per device (a bit of `allowed`) and kernel; any host thread may come first.
template <typename Kernel>
cudaError_t zc_allow_smem(Kernel kernel, int bytes, std::atomic<unsigned long long>* allowed) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (allowed->load(std::memory_order_acquire) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) allowed->fetch_or(bit, std::memory_order_release);
  return e;
}

// Kernels of this file's users come one behind the other, many of them of a few microseconds: each is launched while
// the one before still runs, and waits, before its first access to global memory, until that one has completed
// (their inputs are not declared __restrict__: a read of constant memory might be moved ahead of the wait).
// Calls one after the other: 2 to 4 us each of launch and prologue less (write of 8 x 4096 rows 43.0 -> 40.7 us, read
// 45.4 -> 43.2, windowed single tokens 50.4 -> 48.2, windowed chunks 102 -> 98).
__device__ __forceinline__ void zc_let_next_start() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }
__device__ __forceinline__ void zc_wait_for_last() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
template <typename... KArgs, typename... Args>
cudaError_t zc_launch_early(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

}  // namespace
