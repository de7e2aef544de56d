// What the entry points of every source file share: launch status, checks of pointers and strides, LDS attributes.
#pragma once
#include "../../include/spark_mha.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <atomic>

#include "tiles_gfx950.hpp"

namespace {

using namespace spark;

// hipGetLastError() == hipSuccess, and with SPARK_MHA_DEBUG set in the environment the runtime's own
// description of a failure on stderr (the C ABI itself only returns SPARK_ERR_LAUNCH).
bool launch_ok(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return true;
  static const bool verbose = getenv("SPARK_MHA_DEBUG") != nullptr;
  if (verbose) fprintf(stderr, "spark_mha: %s: %s\n", what, hipGetErrorString(e));
  return false;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A strided tensor is usable if rows hold d contiguous elements, every stride keeps 16-byte
// alignment, and one head's rows span less than 4 GiB (the kernels address a head through a
// 32-bit buffer descriptor).
// An output tensor must in addition give every (batch, head) its own rows: a zero batch or head stride
// (a broadcast, fine for an input) would make all those workgroups store to the same memory.
int check_strides(const spark_strides_t* s, int N, int d, TensorMap* out, bool is_output = false, int B = 1,
                  int H = 1) {
  if (!s) return SPARK_ERR_NULL;
  if (s->batch < 0 || s->head < 0 || s->row < d) return SPARK_ERR_SHAPE;
  if (is_output && ((B > 1 && s->batch == 0) || (H > 1 && s->head == 0))) return SPARK_ERR_SHAPE;
  if ((s->batch | s->head | s->row) & 7) return SPARK_ERR_ALIGN;
  // 31-bit byte offsets inside one head, including the rows a ragged last tile reaches past N
  // (offsets from 2^31 on are how the kernels mark chunks that must read as zeros)
  if ((int64_t)(N + 256) * s->row * 2 >= (int64_t)1 << 31) return SPARK_ERR_SHAPE;
  *out = TensorMap{s->batch, s->head, s->row};
  return SPARK_OK;
}

template <typename KernelT>
int set_smem(KernelT kernel, int bytes) {
  // The kernels address LDS from 0 (lds_origin): that holds only without static LDS in front.
  hipFuncAttributes fa;
  if (hipFuncGetAttributes(&fa, reinterpret_cast<const void*>(kernel)) != hipSuccess || fa.sharedSizeBytes != 0) {
    if (getenv("SPARK_MHA_DEBUG")) fprintf(stderr, "spark_mha: kernel attributes unavailable or static LDS present\n");
    return SPARK_ERR_LAUNCH;
  }
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess && getenv("SPARK_MHA_DEBUG"))
    fprintf(stderr, "spark_mha: hipFuncSetAttribute(%d bytes of LDS): %s\n", bytes, hipGetErrorString(e));
  return e == hipSuccess ? SPARK_OK : SPARK_ERR_LAUNCH;
}

// set_smem once per kernel and device: the attribute belongs to the function on the current
// device, so a process that drives several GPUs needs it on each of them.  `done` holds one bit
// per device ordinal; a failure is not remembered, the next call tries again.
template <typename KernelT>
int ensure_smem(KernelT kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return SPARK_ERR_LAUNCH;
  if (dev < 64 && ((done.load(std::memory_order_acquire) >> dev) & 1u)) return SPARK_OK;
  const int rc = set_smem(kernel, bytes);
  if (rc == SPARK_OK && dev < 64) done.fetch_or(uint64_t(1) << dev, std::memory_order_release);
  return rc;
}

}  // namespace
