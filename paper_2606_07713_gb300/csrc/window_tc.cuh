// What the tcgen05 kernels of windowed attention and of its gradients share: TMA loads and tensor maps of more than
// three dimensions, and masks of bits.
#pragma once
#include <cuda.h>
#include <cstddef>
#include <cstdint>

namespace moa {

// Map over a bf16 tensor of 2 to 5 dimensions, the innermost contiguous; sizes and the box from the
// innermost on, strides in bytes from the second on.  128-byte swizzle, zeros past the end (window_map.cu).
bool encode_bf16_map_nd(CUtensorMap* map, const void* base, int rank, const uint64_t* dims, const uint64_t* strides,
                        const uint32_t* box, char* msg, size_t msglen);

namespace win {

// A tensor's stride as a tensor map has it: positive, whole 16 bytes, below 2^40 bytes.
inline bool describable(int64_t stride, int64_t size) { return size == 1 || (stride > 0 && stride < (int64_t(1) << 39)); }
inline uint64_t map_stride(int64_t stride, int64_t size) { return size == 1 ? 16 : uint64_t(stride) * 2; }

#ifdef __CUDACC__
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t c0,
                                            int32_t c1, int32_t c2, int32_t c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t c0,
                                            int32_t c1, int32_t c2, int32_t c3, int32_t c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
// Bits 32 w .. 32 w + 31 of the number with the lowest x bits set.
__device__ __forceinline__ uint32_t below(int x, int w) {
  const int n = x - 32 * w;
  return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}
#endif

}  // namespace win
}  // namespace moa
