// Which pages a token attends: bounds of the pages' rows of K, a score of every page, and the pages that score highest.
//
// A workgroup takes kChunkPages pages of a (sequence, KV head) pair: the bounds of those that hold new rows are made, then every page is scored; the
// workgroup that is done last for its pair (a ticket) finds the budget-th largest score by digits and lists what lies above, in order.  Scores are summed in 64 bits
// and rounded once, so that pages rank the same however their sums are split; what is equal after that ranks by page.
#include <algorithm>

#include "paged_device.h"

namespace spanattn {

namespace {

constexpr int kSelectThreads = 256, kSelectWaves = 4;
constexpr int kWavePages = 8, kChunkPages = kWavePages * kSelectWaves;

struct SelectArgs {
  const void* q;
  const u32x4* k;
  u32x4* bounds;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* since;  // or null
  int32_t* selected;
  float* scores;         // [batch, kv head, table_pages]
  uint32_t* counters;
  int32_t kv_heads, group, table_pages, page_shift, num_pages, max_len, budget, sinks, recent, counter_stride;
};

// A score's rank as bits: of numbers their order (both zeros alike), NaN above infinity.
__device__ __forceinline__ uint32_t rank_of(float score) {
  const float s = score + 0.f;
  const uint32_t u = __builtin_bit_cast(uint32_t, s);
  if (s != s) return 0xfffffffeu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ double wave_xor(double x, int lanes) { return __shfl_xor(x, lanes, 64); }

template <class Elt, int D>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;  // pieces of a row
  constexpr int kLanes = 2 * kRow;                     // of a page's bounds: 16, 32 or 64
  constexpr int kAtOnce = 64 / kLanes;                 // pages that a wave scores together
  __shared__ int s_bins[256];
  __shared__ int s_wave[2][kSelectWaves];
  __shared__ int s_pick[2];
  __shared__ uint32_t s_ticket;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.y, b = blockIdx.z;
  const size_t bh = (size_t)b * a.kv_heads + h;
  const int len = clampi(a.ctx_lens[b], 0, a.max_len), P = 1 << a.page_shift;
  const int since = clampi(a.since != nullptr ? a.since[b] : a.ctx_lens[b] - 1, 0, len);
  const int pages = (len + P - 1) >> a.page_shift;
  const int chunk0 = (int)blockIdx.x * kChunkPages;
  if (chunk0 >= max(pages, 1)) return;
  const int chunk1 = min(chunk0 + kChunkPages, pages);
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;
  auto bounds_of = [&](int page) { return a.bounds + ((size_t)page * (size_t)a.kv_heads + (size_t)h) * (size_t)kLanes; };

  // ---- bounds of pages with new rows: a wave each, row by row --------------------------------------------
  const int fresh0 = max(chunk0, since >> a.page_shift);
  for (int j = fresh0 + wave; j < chunk1; j += kSelectWaves) {
    const int page = __builtin_amdgcn_readfirstlane(table[j]);
    if ((uint32_t)page >= (uint32_t)a.num_pages) continue;
    const int row0 = max(since - (j << a.page_shift), 0), row1 = min(len - (j << a.page_shift), P);
    if (row0 >= row1) continue;
    constexpr int kRows = 64 / kRow;
    const int piece = lane % kRow;
    const u32x4* rows = a.k + (((size_t)page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) * (size_t)kRow + piece;
    float lo[kPer], hi[kPer];
    if (row0 > 0) {
      Elt::unpack(bounds_of(page)[piece], lo);
      Elt::unpack(bounds_of(page)[kRow + piece], hi);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
    }
    constexpr int kAhead = 4;
    for (int r = row0; r < row1; r += kRows * kAhead) {
      u32x4 x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) x[k] = rows[(size_t)min(r + k * kRows + lane / kRow, row1 - 1) * (size_t)kRow];  // (past the end: the last row again)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float f[kPer];
        Elt::unpack(x[k], f);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          lo[i] = __builtin_elementwise_minimum(lo[i], f[i]);  // (NaN stays)
          hi[i] = __builtin_elementwise_maximum(hi[i], f[i]);
        }
      }
    }
#pragma unroll
    for (int apart = kRow; apart < 64; apart *= 2) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        lo[i] = __builtin_elementwise_minimum(lo[i], __shfl_xor(lo[i], apart, 64));
        hi[i] = __builtin_elementwise_maximum(hi[i], __shfl_xor(hi[i], apart, 64));
      }
    }
    if (lane < kRow) {
      u32x4 l, u;
      if constexpr (Elt::kBytes == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = __builtin_bit_cast(uint32_t, lo[i]), u[i] = __builtin_bit_cast(uint32_t, hi[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = Elt::pack2(lo[2 * i], lo[2 * i + 1]), u[i] = Elt::pack2(hi[2 * i], hi[2 * i + 1]);
      }
      bounds_of(page)[piece] = l;
      bounds_of(page)[kRow + piece] = u;
    }
  }

  int32_t* list = a.selected + bh * (size_t)a.budget;
  if (pages <= a.budget) {  // all of them
    if (chunk0 == 0) {
      for (int i = tid; i < a.budget; i += kSelectThreads) list[i] = i < pages ? i : -1;
    }
    return;
  }

  // ---- scores --------------------------------------------------------------------------------------------
  // The lanes of a page's lower half hold the least values, which meet the queries' negative parts, the others the largest and the positive ones.
  double part[kPer];
  {
    const int piece = lane % kRow;
    const bool upper = lane % kLanes >= kRow;
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[i] = 0.0;
    for (int g = 0; g < a.group; ++g) {
      float f[kPer];
      Elt::unpack(((const u32x4*)a.q)[(bh * (size_t)a.group + (size_t)g) * (size_t)kRow + piece], f);
#pragma unroll
      for (int i = 0; i < kPer; ++i) part[i] += (double)(upper ? __builtin_elementwise_maximum(f[i], 0.f) : __builtin_elementwise_minimum(f[i], 0.f));
    }
  }
  __syncthreads();  // the new bounds are written
  float* scores = a.scores + bh * (size_t)a.table_pages;
  for (int j0 = chunk0 + wave * kWavePages; j0 < min(chunk0 + (wave + 1) * kWavePages, chunk1); j0 += kAtOnce) {
    const int j = min(j0 + lane / kLanes, chunk1 - 1);
    const int page = table[j];
    const bool there = (uint32_t)page < (uint32_t)a.num_pages;
    float f[kPer];
    Elt::unpack(bounds_of(there ? page : 0)[lane % kLanes], f);
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s = fma(part[i], (double)f[i], s);
#pragma unroll
    for (int apart = 1; apart < kLanes; apart *= 2) s += wave_xor(s, apart);
    if (lane % kLanes == 0 && j0 + lane / kLanes < chunk1) publish(scores + j, there ? (float)s : -INFINITY);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // my published scores are acknowledged
  __syncthreads();
  uint32_t* counter = a.counters + bh * (size_t)a.counter_stride;
  const uint32_t chunks = (uint32_t)(pages + kChunkPages - 1) / kChunkPages;
  if (tid == 0) s_ticket = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_ticket != chunks - 1u) return;
  if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // ---- the budget highest ----------------------------------------------------------------------------------
  const int first = min((a.sinks + P - 1) >> a.page_shift, pages), last = max(len - max(a.recent, 1), 0) >> a.page_shift;
  auto key_of = [&](int j) {
    const float s = __hip_atomic_load(scores + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return j < first || j >= last ? 0xffffffffu : rank_of(s);
  };
  uint32_t found = 0;   // digits of the budget-th largest key so far
  int above = 0;        // keys above all that begin so
  for (int shift = 24; shift >= 0; shift -= 8) {
    s_bins[tid] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    for (int j = tid; j < pages; j += kSelectThreads) {
      const uint32_t key = key_of(j);
      if ((key & mask) == found) atomicAdd(&s_bins[key >> shift & 255u], 1);
    }
    __syncthreads();
    // bins from the top: thread t has bin 255 - t
    const int n = s_bins[255 - tid];
    const int incl = wave_inclusive_scan(n);
    if (lane == 63) s_wave[0][wave] = incl;
    __syncthreads();
    int before = above;
    for (int w = 0; w < wave; ++w) before += s_wave[0][w];
    if (before + incl >= a.budget && before + incl - n < a.budget) {
      s_pick[0] = 255 - tid;
      s_pick[1] = before + incl - n;
    }
    __syncthreads();
    found |= (uint32_t)s_pick[0] << shift;
    above = s_pick[1];
  }
  // all above it, and of the equal ones the first: each wave has a run of pages, in order
  const int equal = a.budget - above;
  const int run = ((pages + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, run0 = min(wave * run, pages), run1 = min(run0 + run, pages);
  int more = 0, same = 0;
  for (int j0 = run0; j0 < run1; j0 += 64) {
    const uint32_t key = j0 + lane < run1 ? key_of(j0 + lane) : 0u;
    more += __popcll(__builtin_amdgcn_ballot_w64(j0 + lane < run1 && key > found));
    same += __popcll(__builtin_amdgcn_ballot_w64(j0 + lane < run1 && key == found));
  }
  __syncthreads();
  if (lane == 0) s_wave[0][wave] = more, s_wave[1][wave] = same;
  __syncthreads();
  int more_before = 0, same_before = 0;
  for (int w = 0; w < wave; ++w) more_before += s_wave[0][w], same_before += s_wave[1][w];
  const uint64_t below = (1ull << lane) - 1ull;
  for (int j0 = run0; j0 < run1; j0 += 64) {
    const uint32_t key = j0 + lane < run1 ? key_of(j0 + lane) : 0u;
    const uint64_t up = __builtin_amdgcn_ballot_w64(j0 + lane < run1 && key > found), eq = __builtin_amdgcn_ballot_w64(j0 + lane < run1 && key == found);
    const int m = more_before + __popcll(up & below), s = same_before + __popcll(eq & below);
    if ((up >> lane & 1u) || ((eq >> lane & 1u) && s < equal)) list[m + min(s, equal)] = j0 + lane;
    more_before += __popcll(up);
    same_before += __popcll(eq);
  }
}

}  // namespace
}  // namespace spanattn

extern "C" int paged_select(const span_paged_desc_t* desc, const void* q, const void* k_pages, void* bounds, const int32_t* block_table,
                            const int32_t* ctx_lens, const int32_t* since, int32_t* selected) {
  using namespace spanattn;
  int rc = check_paged(desc);
  if (rc != SPAN_OK) return rc;
  rc = check_select(desc);
  if (rc != SPAN_OK) return rc;
  if (!q || !k_pages || !bounds || !block_table || !ctx_lens || !selected) return SPAN_ERR_NULL;
  const size_t need = select_workspace(desc);
  if (!desc->workspace || ((uintptr_t)desc->workspace & 255u) || desc->workspace_bytes < need) return SPAN_ERR_WORKSPACE;
  SelectArgs a = {};
  a.q = q;
  a.k = (const u32x4*)k_pages;
  a.bounds = (u32x4*)bounds;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.since = since;
  a.selected = selected;
  a.scores = (float*)((char*)desc->workspace + counter_bytes(desc));
  a.counters = (uint32_t*)desc->workspace;
  a.counter_stride = (int32_t)(counter_bytes(desc) / sizeof(int32_t) / ((size_t)desc->batch * desc->kv_heads));
  a.kv_heads = desc->kv_heads;
  a.group = desc->heads / desc->kv_heads;
  a.table_pages = desc->table_pages;
  a.page_shift = page_shift(desc);
  a.num_pages = desc->num_pages;
  a.max_len = capacity(desc);
  a.budget = desc->budget;
  a.sinks = std::min(desc->sinks, a.max_len);
  a.recent = std::min(desc->recent, a.max_len);
  const dim3 grid((unsigned)((desc->table_pages + kChunkPages - 1) / kChunkPages), (unsigned)desc->kv_heads, (unsigned)desc->batch);
  const bool d128 = desc->head_dim == 128;
  hipStream_t stream = (hipStream_t)desc->stream;
  auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kSelectThreads), 0, stream, a); };
  switch (desc->dtype) {
    case SPAN_F32:
      d128 ? start(select_kernel<F32, 128>) : start(select_kernel<F32, 64>);
      break;
    case SPAN_F16:
      d128 ? start(select_kernel<F16, 128>) : start(select_kernel<F16, 64>);
      break;
    default:
      d128 ? start(select_kernel<BF16, 128>) : start(select_kernel<BF16, 64>);
  }
  return launched();
}
