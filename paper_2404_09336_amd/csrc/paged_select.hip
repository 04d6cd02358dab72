// Which pages a token attends: bounds of the pages' rows of K, a score of every page, and the pages that score highest.
//
// A workgroup takes `chunk` pages of a (sequence, KV head) pair: the bounds of those that hold new rows are made, then every page is scored.  Where one workgroup has all of a pair's pages the
// scores stay in LDS, otherwise the workgroup that is done last for its pair (a ticket) fetches them; it finds the budget-th largest by digits and lists what lies above, in order.
// Scores are summed in 64 bits and rounded once, so that pages rank the same however their sums are split; what is equal after that ranks by page.
// What bounds it: memory, 2 * head_dim values of bounds a page, and behind it some 7 us of a launch, the first trips and the selection.  64 x 8 pairs of 2000 .. 8192 positions in pages of 16, four query heads
// each, fp16 (85 MB): 21.8 us; twice the pages take 13 more, 6.5 TB/s.  The bounds of 4 x 8 prompts of 8000 .. 32768 in pages of 64, bf16 (156 MB of K): 37.5 us, of which the rows take 28.
// Digits of 8 bits: four rounds of counting at most, fewer where a digit ends with the list full, two barriers each.
#include <algorithm>

#include "paged_device.h"

namespace spanattn {

namespace {

constexpr int kSelectThreads = 512, kSelectWaves = 8;
constexpr int kChunkMost = 2048, kChunkLeast = 16;        // pages of a workgroup
constexpr int kHeldKeys = 4, kHeldPages = kHeldKeys * kSelectThreads;
// A call aims at so many workgroups, one for each pair where there are as many.  us, 512 -> 1024 (a wave of 256 threads less -> 256 threads): 64 x 8 pairs of 2000 .. 8192 positions in pages of 16 22.6 -> 31.0
// (25.3); 4 x 8 of 8000 .. 32768 in pages of 64, all bounds made, 38.0 -> 42.8 (39.8).  The next group's bounds asked for ahead of a group's sums: 23.6 and 38.1.
constexpr int64_t kSelectWorkgroups = 512;

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
  int32_t kv_heads, group, table_pages, page_shift, num_pages, max_len, budget, sinks, recent, counter_stride, chunk;
};

// A score's rank as bits: of numbers their order (both zeros alike), NaN above infinity.
__device__ __forceinline__ uint32_t rank_of(float score) {
  const float s = score + 0.f;
  const uint32_t u = __builtin_bit_cast(uint32_t, s);
  if (s != s) return 0xfffffffeu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// x of the lane `kApart` further in its numbers' bits.
template <int kApart>
__device__ __forceinline__ uint32_t from_apart(uint32_t x) {
  if constexpr (kApart == 1) return (uint32_t)dpp_i<0xB1>((int)x);  // quad_perm [1,0,3,2]
  else if constexpr (kApart == 2) return (uint32_t)dpp_i<0x4E>((int)x);  // quad_perm [2,3,0,1]
  else if constexpr (kApart == 4) {
    const int up = __builtin_amdgcn_update_dpp((int)x, (int)x, 0x104, 0xf, 0x5, false);  // row_shl:4, the first and third four of a row
    return (uint32_t)__builtin_amdgcn_update_dpp(up, (int)x, 0x114, 0xf, 0xa, false);    // row_shr:4, the others
  } else {
    static_assert(kApart == 8, "within a row of 16 lanes");
    return (uint32_t)dpp_i<0x128>((int)x);  // row_ror:8
  }
}

// Sums of two values over lanes kApart apart: the lanes whose number has that bit clear get low's, the others high's.
template <int kApart>
__device__ __forceinline__ double add_apart(double low, double high, int lane) {
  const u32x2 l = __builtin_bit_cast(u32x2, low), h = __builtin_bit_cast(u32x2, high);
  u32x2 a, b;
  if constexpr (kApart >= 16) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (kApart == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(l[i], h[i], false, false);
        a[i] = r[0];
        b[i] = r[1];
      } else {
        const auto r = __builtin_amdgcn_permlane32_swap(l[i], h[i], false, false);
        a[i] = r[0];
        b[i] = r[1];
      }
    }
  } else {
    const bool upper = lane & kApart;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      a[i] = upper ? h[i] : l[i];
      b[i] = from_apart<kApart>(upper ? l[i] : h[i]);
    }
  }
  return __builtin_bit_cast(double, a) + __builtin_bit_cast(double, b);
}

// Eight values a lane, over aligned groups of kLanes lanes: lane i ends with the sum of value number i / (kLanes / 8) of its group, the same in all lanes of that number.
template <int kLanes>
__device__ __forceinline__ double sum_of_eight(double (&s)[8], int lane) {
  double four[4], two[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) four[i] = add_apart<kLanes / 2>(s[i], s[i + 4], lane);
#pragma unroll
  for (int i = 0; i < 2; ++i) two[i] = add_apart<kLanes / 4>(four[i], four[i + 2], lane);
  double one = add_apart<kLanes / 8>(two[0], two[1], lane);
  if constexpr (kLanes == 64) one = add_apart<4>(one, one, lane);
  if constexpr (kLanes >= 32) one = add_apart<2>(one, one, lane);
  return add_apart<1>(one, one, lane);
}

template <class Elt, int D>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const SelectArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;  // pieces of a row
  constexpr int kLanes = 2 * kRow;                     // of a page's bounds: 16, 32 or 64
  constexpr int kAtOnce = 64 / kLanes;                 // pages of one load
  constexpr int kGroup = 8 * kAtOnce;                  // ... that a wave scores together
  __shared__ __attribute__((aligned(16))) int s_bins[2][256];  // of this digit, and of the next
  __shared__ int s_wave[2][kSelectWaves];
  __shared__ int s_pick[3];
  __shared__ uint32_t s_ticket;
  __shared__ float s_scores[kChunkMost];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.y, b = blockIdx.z;
  if (tid < 256) s_bins[0][tid] = 0;
  const size_t bh = (size_t)b * a.kv_heads + h;
  const int len = clampi(a.ctx_lens[b], 0, a.max_len), P = 1 << a.page_shift;
  const int since = clampi(a.since != nullptr ? a.since[b] : a.ctx_lens[b] - 1, 0, len);
  const int pages = (len + P - 1) >> a.page_shift;
  const int chunk0 = (int)blockIdx.x * a.chunk;
  if (chunk0 >= max(pages, 1)) return;
  const int chunk1 = min(chunk0 + a.chunk, pages);
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;
  auto bounds_of = [&](int page) { return a.bounds + ((size_t)page * (size_t)a.kv_heads + (size_t)h) * (size_t)kLanes; };
  // pages ahead of `first` and from `last` on are listed in any case
  const int first = min((a.sinks + P - 1) >> a.page_shift, pages), last = max(len - max(a.recent, 1), 0) >> a.page_shift;

  const bool scored = pages > a.budget, alone = pages <= a.chunk;
  float* scores = a.scores + bh * (size_t)a.table_pages;
  auto put_score = [&](int j, float score) {
    if (alone) s_scores[j] = score;
    else publish(scores + j, score);
  };
  // The lanes of a page's lower half hold the least values, which meet the queries' negative parts, the others the largest and the positive ones.
  double part[kPer];
  {
    const int piece = lane % kRow;
    const bool upper = lane % kLanes >= kRow;
#pragma unroll
    for (int i = 0; i < kPer; ++i) part[i] = 0.0;
    for (int g = 0; g < (scored ? a.group : 0); ++g) {
      float f[kPer];
      Elt::unpack(((const u32x4*)a.q)[(bh * (size_t)a.group + (size_t)g) * (size_t)kRow + piece], f);
#pragma unroll
      for (int i = 0; i < kPer; ++i) part[i] += (double)(upper ? __builtin_elementwise_maximum(f[i], 0.f) : __builtin_elementwise_minimum(f[i], 0.f));
    }
  }

  // ---- bounds, and scores, of pages with new rows: a wave each, row by row -------------------------------
  const int fresh0 = max(chunk0, since >> a.page_shift);
  for (int j = fresh0 + wave; j < chunk1; j += kSelectWaves) {
    const int page = __builtin_amdgcn_readfirstlane(table[j]);
    if ((uint32_t)page >= (uint32_t)a.num_pages) {
      if (scored && lane == 0) put_score(j, -INFINITY);
      continue;
    }
    const int row0 = max(since - (j << a.page_shift), 0), row1 = min(len - (j << a.page_shift), P);  // (since = len at the page's end: none)
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
    constexpr int kAhead = 8;
    for (int r = row0; r < row1; r += kRows * kAhead) {
      u32x4 x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)  // (past the end: the last row again)
        x[k] = __builtin_nontemporal_load(rows + (size_t)min(r + k * kRows + lane / kRow, row1 - 1) * (size_t)kRow);
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
    if (scored) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) s = fma(part[i], (double)(lane % kLanes >= kRow ? hi[i] : lo[i]), s);
#pragma unroll
      for (int apart = 1; apart < kLanes; apart *= 2) s += __shfl_xor(s, apart, 64);
      if (lane == 0) put_score(j, (float)s);
    }
  }

  int32_t* list = a.selected + bh * (size_t)a.budget;
  if (!scored) {  // all of them
    if (chunk0 == 0) {
      for (int i = tid; i < a.budget; i += kSelectThreads) list[i] = i < pages ? i : -1;
    }
    return;
  }

  // ---- scores of the others -----------------------------------------------------------------------------
  const int old1 = min(chunk1, fresh0);
  // a group's pages in the first lanes, the next group's on their way
  auto entry_of = [&](int j0) { return lane < kGroup && j0 + lane < old1 ? table[j0 + lane] : -1; };
  int j0 = chunk0 + wave * kGroup;
  int entry = entry_of(j0);
  for (; j0 < old1; j0 += kSelectWaves * kGroup) {
    const uint64_t there = __builtin_amdgcn_ballot_w64((uint32_t)entry < (uint32_t)a.num_pages);
    const int safe = (uint32_t)entry < (uint32_t)a.num_pages ? entry : 0;
    u32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __builtin_nontemporal_load(bounds_of(__shfl(safe, k * kAtOnce + lane / kLanes)) + lane % kLanes);
    entry = entry_of(j0 + kSelectWaves * kGroup);
    double s[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float f[kPer];
      Elt::unpack(x[k], f);
      s[k] = 0.0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) s[k] = fma(part[i], (double)f[i], s[k]);
    }
    const double sum = sum_of_eight<kLanes>(s, lane);
    const int mine = lane % kLanes / (kLanes / 8) * kAtOnce + lane / kLanes;  // of the group's pages
    if (lane % (kLanes / 8) == 0 && j0 + mine < old1) put_score(j0 + mine, there >> mine & 1u ? (float)sum : -INFINITY);
  }
  if (alone) {
    __syncthreads();
  } else {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // my published scores are acknowledged
    __syncthreads();
    uint32_t* counter = a.counters + bh * (size_t)a.counter_stride;
    const uint32_t chunks = (uint32_t)((pages + a.chunk - 1) / a.chunk);
    if (tid == 0) s_ticket = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (s_ticket != chunks - 1u) return;
    if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }

  // ---- the budget highest ----------------------------------------------------------------------------------
  // Each wave has a run of pages, in order; of up to kHeldPages their keys stay in registers.
  const int run = ((pages + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64, run0 = min(wave * run, pages), run1 = min(run0 + run, pages);
  auto key_of = [&](int j) {
    if (j >= run1) return 0u;  // (no page's)
    if (j < first || j >= last) return 0xffffffffu;
    return rank_of(alone ? s_scores[j] : __hip_atomic_load(scores + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  };
  const bool held = pages <= kHeldPages;
  uint32_t keys[kHeldKeys];
#pragma unroll
  for (int i = 0; i < kHeldKeys; ++i) keys[i] = held ? key_of(run0 + 64 * i + lane) : 0u;
  auto each = [&](auto&& f) {  // f(page of lane 0, this lane's key), in order
    if (held) {
#pragma unroll
      for (int i = 0; i < kHeldKeys; ++i) {
        if (run0 + 64 * i < run1) f(run0 + 64 * i, keys[i]);
      }
    } else {
      for (int j = run0; j < run1; j += 64) f(j, key_of(j + lane));
    }
  };
  uint32_t found = 0;    // digits of the budget-th largest key so far
  int above = 0;         // keys above all that begin so
  bool all = false;      // ... and those are listed too
  for (int shift = 24, buffer = 0; shift >= 0 && !all; shift -= 8, buffer ^= 1) {
    const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
    each([&](int, uint32_t key) {
      if (key != 0u && (key & mask) == found) atomicAdd(&s_bins[buffer][key >> shift & 255u], 1);
    });
    __syncthreads();
    if (wave == 0) {  // bins from the top: lane l has 255 - 4 l and the three below
      const i32x4 n = *reinterpret_cast<const i32x4*>(&s_bins[buffer][252 - 4 * lane]);
      int before = above + wave_inclusive_scan(n[0] + n[1] + n[2] + n[3]) - (n[0] + n[1] + n[2] + n[3]);
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        if (before < a.budget && before + n[k] >= a.budget) {
          s_pick[0] = 252 - 4 * lane + k;
          s_pick[1] = before;
          s_pick[2] = before + n[k] == a.budget;
        }
        before += n[k];
      }
    } else if (tid < 64 + 256) {
      s_bins[buffer ^ 1][tid - 64] = 0;
    }
    __syncthreads();
    found |= (uint32_t)s_pick[0] << shift;
    above = s_pick[1];
    all = s_pick[2] != 0;
  }
  // listed: keys above `found`, and of those equal to it the first; where a digit ended with the list full, all from `found` on
  const int equal = all ? 0 : a.budget - above;
  auto over = [&](uint32_t key) { return key > found || (all && key == found); };
  int more = 0, same = 0;
  each([&](int, uint32_t key) {
    more += __popcll(__builtin_amdgcn_ballot_w64(key != 0u && over(key)));
    same += __popcll(__builtin_amdgcn_ballot_w64(key == found));
  });
  if (lane == 0) s_wave[0][wave] = more, s_wave[1][wave] = same;
  __syncthreads();
  int more_before = 0, same_before = 0;
  for (int w = 0; w < wave; ++w) more_before += s_wave[0][w], same_before += s_wave[1][w];
  const uint64_t below = (1ull << lane) - 1ull;
  each([&](int j, uint32_t key) {
    const uint64_t up = __builtin_amdgcn_ballot_w64(key != 0u && over(key)), eq = __builtin_amdgcn_ballot_w64(key != 0u && key == found);
    const int m = more_before + __popcll(up & below), e = min(same_before + __popcll(eq & below), equal);
    if ((up >> lane & 1u) || ((eq >> lane & 1u) && e < equal)) list[m + e] = j + lane;
    more_before += __popcll(up);
    same_before += __popcll(eq);
  });
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
  const int64_t pairs = (int64_t)desc->batch * desc->kv_heads, per_pair = std::max<int64_t>(1, kSelectWorkgroups / pairs);
  const int64_t chunk = (desc->table_pages + per_pair - 1) / per_pair;
  a.chunk = (int32_t)std::min<int64_t>(std::max<int64_t>((chunk + 15) / 16 * 16, kChunkLeast), kChunkMost);
  const dim3 grid((unsigned)((desc->table_pages + a.chunk - 1) / a.chunk), (unsigned)desc->kv_heads, (unsigned)desc->batch);
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
