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

// Positions that the token at position n - 1 sees: [0, sinks) and from `low` on, of those below n that the table has.
struct Seen {
  int sinks, low, count;
};
__device__ __forceinline__ Seen seen_by_last(int n, int max_len, int window, int sinks) {
  const int held = clampi(n, 0, max_len);
  Seen s;
  s.low = window > 0 ? clampi(max(n, 0) - window, 0, held) : 0;
  s.sinks = min(sinks, s.low);
  s.count = held - s.low + s.sinks;
  return s;
}

}  // namespace spanattn
#endif
