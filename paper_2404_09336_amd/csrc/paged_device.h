// Device code shared by the kernels on a cache in pages.
#ifndef PAGED_DEVICE_H_
#define PAGED_DEVICE_H_

#include "paged_internal.h"
#include "span_device.h"

namespace spanattn {

// What an entry point returns after a launch.
inline int launched() {
  const hipError_t err = hipGetLastError();
  if (err == hipSuccess) return SPAN_OK;
  g_last_hip_error = (int)err;
  return SPAN_ERR_HIP;
}

// Memory reached through 64-bit addresses (a pool is larger than what a buffer descriptor spans), as global and not flat accesses.
#define SPAN_GLOBAL __attribute__((address_space(1)))
typedef const SPAN_GLOBAL u32x4* global_u32x4;
typedef const SPAN_GLOBAL u32x2* global_u32x2;

// Where position p of a sequence lies in the pool: number of its row among those of one head (page * page_size + row in the
// page), or -1 if its page is not one of the pool's.
__device__ __forceinline__ int pool_row(const int32_t* table_of_b, int p, int page_shift, int num_pages) {
  const int page = table_of_b[p >> page_shift];
  return (uint32_t)page < (uint32_t)num_pages ? (page << page_shift) + (p & ((1 << page_shift) - 1)) : -1;
}

// The first sequence that ends behind row t, by sixty-fourths of the list: one load per step, one step for up to 64 sequences.
// Returns -1 where there is none.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int batch, int t, int lane) {
  int low = 0, n = batch;
  while (true) {
    const int step = (n + 63) >> 6;
    const bool ended = offsets[low + min((lane + 1) * step, n)] <= t;
    const int past = __popcll(__builtin_amdgcn_ballot_w64(ended)) * step;
    if (past >= n) return -1;
    low += past;
    if (step == 1) return low;
    n = min(step, n - past);
  }
}

}  // namespace spanattn
#endif
