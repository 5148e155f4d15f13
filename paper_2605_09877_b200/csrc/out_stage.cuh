// Staging of output rows in shared memory, for the kernels whose threads hold one row each.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace kvm {

// Output staging: a 128 x D bf16 tile, row-major in shared memory, the 16-byte chunks of a row
// permuted by the row index so that neither the row-per-thread writes nor the row-contiguous reads
// conflict on the banks.
template <int D>
__device__ __forceinline__ uint4* stage_chunk(uint8_t* stage, int row, int k) {
  constexpr int CPR = D / 8;   // chunks per row
  return reinterpret_cast<uint4*>(stage + row * (D * 2) + ((k ^ (row & (CPR - 1))) << 4));
}
// 32 fp32 accumulator values of one row -> four chunks (channels [32 c, 32 c + 32)), scaled
template <int D>
__device__ __forceinline__ void stage_row32(uint8_t* stage, int row, int c, const uint32_t (&r)[32], float inv) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[8 * q + 2 * i]) * inv, __uint_as_float(r[8 * q + 2 * i + 1]) * inv);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *stage_chunk<D>(stage, row, 4 * c + q) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace kvm
