// The keep mask that the dropout kernels regenerate, written out for inspection (spark_dropout_mask).
#pragma once
#include "dropout_gfx950.hpp"

namespace spark {

// The keep mask itself, one byte per entry (1 = keep), [B*H][Nq][Nk]: one thread per 4 x 4 block.
__global__ void dropout_mask_kernel(unsigned char* __restrict__ M, int Nq, int Nk, int qblocks,
                                    int kblocks, long long total_blocks, Dropout dr) {
  const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= total_blocks) return;
  const int jb = (int)(t % kblocks);
  const long long rest = t / kblocks;
  const int ib = (int)(rest % qblocks);
  const int h = (int)(rest / qblocks);
  uint32_t x[4];
  philox4x32_10((uint32_t)jb, (uint32_t)ib, (uint32_t)h, dr.offset, dr.key0, dr.key1, x);
  for (int r = 0; r < 4; ++r) {
    const int i = 4 * ib + r;
    if (i >= Nq) break;
    for (int c = 0; c < 4; ++c) {
      const int j = 4 * jb + c;
      if (j >= Nk) break;
      M[((size_t)h * Nq + i) * Nk + j] = ((x[r] >> (8 * c)) & 0xFFu) >= dr.thr ? 1 : 0;
    }
  }
}

}  // namespace spark
