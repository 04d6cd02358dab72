// What the one-token attention kernels on a cache in pages share: arguments, the slices of a call, and how the states of waves and slices become one.
#ifndef PAGED_ATTEND_H_
#define PAGED_ATTEND_H_

#include "paged_device.h"

namespace spanattn {

struct PagedArgs : LaunchArgs {  // heads: KV heads; max_len: positions of a sequence's table; k, v: the pools
  const int32_t* block_table;
  int32_t table_pages, page_shift, num_pages;
  int32_t group;             // query heads per KV head
  int32_t batch, window, sinks;
  int32_t room, more_room;   // > 0: slices per head aimed at, see slice_length, and rows of the grid; 0: num_splits each, or the table
  int32_t whole;             // up to so many positions a sequence is not cut
  int32_t least;             // positions of a slice at least
  float* scores;             // [batch, kv head, query head of the group, max_len] unscaled scores by virtual position, or null
  float* final_ml;           // [batch, query head] (maximum, sum)
  int32_t* counts;           // span form with weights: [batch] attended positions
  int32_t* list;             // ... and [batch, max_len] the positions themselves
  float* weights;
  const int32_t* selected;   // selected form: [batch, kv head, budget] pages of a sequence
  int32_t budget;
  int32_t weights_here;      // 1: the workgroup that attends adds up the weights too (PagedPlan::own_weights)
};
struct PagedArgsPlain : PagedArgs {
  static constexpr bool kHasTable = false;
};
struct PagedArgsTable : PagedArgs {
  static constexpr bool kHasTable = true;
  uint32_t table[kMaxPlanSlices];  // pack_slice entries
};

// Selected form: positions of a pair as far as the length tells (what a list's entries leave of them is seen row by row), ...
__device__ __forceinline__ int selected_positions(const PagedArgs& a, int len) {
  const int held = clampi(len, 0, a.max_len), page = 1 << a.page_shift;
  return min((held + page - 1) >> a.page_shift, a.budget) << a.page_shift;
}
// ... and the v-th of them, or -1 where the entry is none of the sequence's pages or the sequence ends ahead of the row.
__device__ __forceinline__ int selected_position(const PagedArgs& a, size_t bh, int len, int v) {
  const int page = a.selected[bh * (size_t)a.budget + (size_t)(v >> a.page_shift)];
  if ((uint32_t)page >= (uint32_t)a.table_pages) return -1;
  const int p = (page << a.page_shift) + (v & ((1 << a.page_shift) - 1));
  return p < len ? p : -1;
}

struct Slice {
  int b, split, nsl, y0, len;  // sequence, slice within it, slices of it, slot of its first slice; its length (locate_slice)
};

// The slice that row y of the grid is (slice_length).  Every workgroup works it out for itself: one load of the lengths, which it needs anyway, and a few scans for up to 64 sequences.
// count_of(length): positions that a sequence of so many attends.
template <class CountOf>
__device__ __forceinline__ Slice locate_slice(const PagedArgs& a, int y, int lane, CountOf&& count_of) {
  int len = 0, n = 0;
  auto fetch = [&](int c) {
    len = c + lane < a.batch ? a.ctx_lens[c + lane] : 0;
    n = count_of(len);
  };
  uint32_t all = 0, longest = 1;
  for (int c = 0; c < a.batch; c += 64) {
    fetch(c);
    all += (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_scan(n), 63);
    longest = max(longest, (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_max(n), 63));
  }
  auto slices = [&](uint32_t T) { return n > a.whole ? (int)(((uint32_t)n + T - 1u) / T) : 1; };  // of this lane's sequence
  const uint32_t T = slice_length(all, longest, (uint32_t)a.batch, (uint32_t)a.room, (uint32_t)a.more_room, (uint32_t)a.whole, (uint32_t)a.least, [&](uint32_t T) {  // of all
    uint32_t total = 0;
    for (int c = 0; c < a.batch; c += 64) {
      if (a.batch > 64) fetch(c);
      total += (uint32_t)__builtin_amdgcn_readlane(wave_inclusive_scan(c + lane < a.batch ? slices(T) : 0), 63);
    }
    return total;
  });
  Slice s = {-1, 0, 1, 0, 0};
  int before = 0;
  for (int c = 0; c < a.batch; c += 64) {
    if (a.batch > 64) fetch(c);
    const int nsl = c + lane < a.batch ? slices(T) : 0;
    const int incl = before + wave_inclusive_scan(nsl);
    const uint64_t past = __builtin_amdgcn_ballot_w64(incl > y);
    if (past != 0) {
      const int at = (int)__builtin_ctzll(past);
      s.b = c + at;
      s.nsl = __builtin_amdgcn_readlane(nsl, at);
      s.y0 = __builtin_amdgcn_readlane(incl, at) - s.nsl;
      s.split = y - s.y0;
      s.len = __builtin_amdgcn_readlane(len, at);
      break;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return s;
}

// A wave's instruction priority falls as it gets on with its rows.  Among equals a SIMD issues the oldest wave first, and the workgroups that arrive last on
// a CU got their first rows when the others were nearly done (stamps: after 5 to 67 us of a call of 107), to end alone.  64 x 8 pairs of 512 .. 4096
// 107.1 -> 104.6; smaller calls 0 to 1 %.
__device__ __forceinline__ void priority(int done, int quarter) {
  if (done == 0) __builtin_amdgcn_s_setprio(3);
  else if (done == quarter) __builtin_amdgcn_s_setprio(2);
  else if (done == 2 * quarter) __builtin_amdgcn_s_setprio(1);
  else if (done == 3 * quarter) __builtin_amdgcn_s_setprio(0);
}

// The waves' states are merged in LDS; a slice that is its sequence's only one goes out as it is, others by way of the workspace: the workgroup that arrives last
// for the pair merges them all.  s_ml[j][wave] holds query column j's reference and the sum over the wave; put(acc[wave]) stores the wave's unnormalised outputs, [column][channel], once
// the tables that acc lies over are no longer read; both sums are weight_scale times the weights'.  kFinal: (maximum, sum) go to final_ml.  True for the only slice.
// kTeams: where a group has 16 / kTeams heads at most, so many teams of threads share a pair's slices out (4 x 8 pairs of 8000 .. 32768 positions in 4 bits, up to 25 slices a pair: 26.9 -> 25.2 us; one trip to memory of eight slices each in place of four).
template <int D, bool kFinal, int kTeams, class Put>
__device__ __forceinline__ bool finish_pair(const PagedArgs& a, const Slice& sl, int h, float post, float weight_scale, f32x2 (&s_ml)[16][kWavesPerBlock],
                                            float (&acc)[kWavesPerBlock][16][D + 4], uint32_t& s_ticket, Put&& put) {
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kv_heads = a.heads, group = a.group, split = sl.split, nsl = sl.nsl;
  const size_t bh = (size_t)sl.b * kv_heads + h;
  auto qrow = [&](int j) { return bh * (size_t)group + (size_t)min(j, group - 1); };
  constexpr int kPerToken = kThreads / 16, kQuads = D / 4 / kPerToken;
  const int mine = tid % (kThreads / kTeams) / kPerToken, part = tid % kPerToken;  // query head, share of its quads of columns
  const int team = kTeams == 1 ? 0 : wave / (kWavesPerBlock / kTeams);
  const bool direct = nsl == 1;
  const size_t slot0 = (size_t)sl.y0 * kv_heads + h, my_slot = slot0 + (size_t)split * kv_heads;
  auto acc_slot = [&](size_t slot) { return slab_resource(a.part_acc + slot * (size_t)(group * D), (uint32_t)(group * D) * 4u); };
  auto ml_slot = [&](size_t slot) { return slab_resource(a.part_ml + slot * (size_t)(group * 2), (uint32_t)group * 8u); };
  auto store_row = [&](float M, float L, const f32x4 (&o)[kQuads]) {
    const float sum = L != 0.f ? L : 1.f;
    float* row = a.out + qrow(mine) * D + 4 * part;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) *reinterpret_cast<f32x4*>(row + 4 * kPerToken * i) = f32x4{o[i][0] / sum, o[i][1] / sum, o[i][2] / sum, o[i][3] / sum};
    if (kFinal && part == 0) *reinterpret_cast<f32x2*>(a.final_ml + 2 * qrow(mine)) = f32x2{M, L / weight_scale};
  };
  __syncthreads();  // the (maximum, sum) pairs are in LDS; the streaming tables are no longer read
  put(acc[wave]);
  float M, L;
  f32x4 o[kQuads];
  auto join = [&](auto states) {  // of the first so many waves', or teams', states in LDS
    constexpr int kStates = decltype(states)::value;
    float weight[kStates];
    f32x2 ml[kStates];
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < kStates; ++w) ml[w] = s_ml[mine][w];
#pragma unroll
    for (int w = 0; w < kStates; ++w)
      if (ml[w][1] != 0.f) M = fmaxf(M, ml[w][0]);  // (a NaN sum counts: it has to reach the output)
#pragma unroll
    for (int w = 0; w < kStates; ++w) {
      weight[w] = ml[w][1] != 0.f ? __builtin_amdgcn_exp2f((ml[w][0] - M) * post) : 0.f;
      L = fmaf(weight[w], ml[w][1], L);
    }
    __syncthreads();
    if (mine < group && team == 0) {
#pragma unroll
      for (int i = 0; i < kQuads; ++i) {
        o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kStates; ++w) {
          const f32x4 ow = *reinterpret_cast<const f32x4*>(&acc[w][mine][4 * (part + kPerToken * i)]);
#pragma unroll
          for (int k = 0; k < 4; ++k) o[i][k] = fmaf(weight[w], ow[k], o[i][k]);
        }
      }
    }
  };
  join(std::integral_constant<int, kWavesPerBlock>());
  if (mine < group && team == 0) {
    if (direct) {
      store_row(M, L, o);
    } else {
      const __amdgpu_buffer_rsrc_t slot = acc_slot(my_slot);
#pragma unroll
      for (int i = 0; i < kQuads; ++i) publish4(slot, (uint32_t)(mine * D + 4 * (part + kPerToken * i)) * 4u, o[i]);
      if (part == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{M, L}), ml_slot(my_slot), (uint32_t)mine * 8u, 0, kThrough);
    }
  }
  if (direct) return true;

  // ---- several slices: the workgroup that arrives last for the pair merges them all (the hand-over of matrix_kernel) ----
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // my published stores are acknowledged
  __syncthreads();
  if (tid == 0) s_ticket = (uint32_t)__hip_atomic_fetch_add(a.counters + bh * (size_t)a.counter_stride, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (s_ticket != (uint32_t)(nsl - 1)) return false;
  if (mine < group) {
    constexpr int kMerge = 8;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    M = -INFINITY;
    L = 0.f;
    for (int s0 = team; s0 < nsl; s0 += kTeams * kMerge) {
      f32x2 ml[kMerge];
      f32x4 os[kMerge][kQuads];
#pragma unroll
      for (int k = 0; k < kMerge; ++k) {
        const size_t slot = slot0 + (size_t)min(s0 + kTeams * k, nsl - 1) * kv_heads;  // (past the end: a slot that exists, unused)
        ml[k] = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(ml_slot(slot), (uint32_t)mine * 8u, 0, kThrough));
        const __amdgpu_buffer_rsrc_t states = acc_slot(slot);
#pragma unroll
        for (int i = 0; i < kQuads; ++i) os[k][i] = observe4(states, (uint32_t)(mine * D + 4 * (part + kPerToken * i)) * 4u);
      }
      const float before = M;
#pragma unroll
      for (int k = 0; k < kMerge; ++k) {
        if (s0 + kTeams * k >= nsl) ml[k][1] = 0.f;
        if (ml[k][1] != 0.f) M = fmaxf(M, ml[k][0]);
      }
      const float safe = M == -INFINITY ? 0.f : M;
      if (s0 > team) {
        const float old = __builtin_amdgcn_exp2f((before - safe) * post);
        L *= old;
#pragma unroll
        for (int i = 0; i < kQuads; ++i) o[i] *= old;
      }
#pragma unroll
      for (int k = 0; k < kMerge; ++k) {
        if (s0 + kTeams * k < nsl) {
          const float w = ml[k][1] != 0.f ? __builtin_amdgcn_exp2f((ml[k][0] - safe) * post) : 0.f;
          L = fmaf(w, ml[k][1], L);
#pragma unroll
          for (int i = 0; i < kQuads; ++i) {
#pragma unroll
            for (int c = 0; c < 4; ++c) o[i][c] = fmaf(w, os[k][i][c], o[i][c]);
          }
        }
      }
    }
    if constexpr (kTeams == 1) {
      store_row(M, L, o);
    } else {
      if (part == 0) s_ml[mine][team] = f32x2{M, L};
#pragma unroll
      for (int i = 0; i < kQuads; ++i) *reinterpret_cast<f32x4*>(&acc[team][mine][4 * (part + kPerToken * i)]) = o[i];
    }
  }
  if constexpr (kTeams > 1) {
    __syncthreads();
    join(std::integral_constant<int, kTeams>());
    if (mine < group && team == 0) store_row(M, L, o);
  }
  if (tid == 0) __hip_atomic_store(a.counters + bh * (size_t)a.counter_stride, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return false;
}

// Arguments and plan of a one-token call, or what it is refused with.  `table`: kMaxPlanSlices entries.
inline int one_token_args(const span_paged_desc_t* d, PagedKind kind, const void* q, const void* k, const void* v, const int32_t* block_table,
                          const int32_t* ctx_lens, const int32_t* offsets, const int32_t* starts, const int32_t* ends, const int32_t* selected, float scale,
                          float* weights, float* out, PagedArgs* args, PagedPlan* plan, uint32_t* table, bool fp4 = false) {
  const bool spans = kind == kPagedSpans;
  const int rc = check_paged(d);
  if (rc != SPAN_OK) return rc;
  if (!q || !k || !v || !block_table || !out) return SPAN_ERR_NULL;
  if (spans ? !offsets || (d->num_intervals > 0 && (!starts || !ends)) : !ctx_lens) return SPAN_ERR_NULL;
  if (kind == kPagedSelected && (d->budget < 1 || !selected)) return d->budget < 1 ? SPAN_ERR_SHAPE : SPAN_ERR_NULL;
  const PagedPlan& p = *plan;
  *plan = plan_paged(d, kind, table, fp4);
  const PagedWorkspace w = paged_workspace(d, p, kind, weights != nullptr);
  if (w.total > 0 && (!d->workspace || ((uintptr_t)d->workspace & 255u) || d->workspace_bytes < w.total)) return SPAN_ERR_WORKSPACE;
  char* at = (char*)d->workspace;
  PagedArgs& a = *args;
  a = PagedArgs{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.offsets = offsets;
  a.starts = starts;
  a.ends = ends;
  a.ctx_lens = ctx_lens;
  a.counters = w.sliced ? (int32_t*)at : nullptr;
  a.counter_stride = (int32_t)(counter_bytes(d) / sizeof(int32_t) / ((size_t)d->batch * d->kv_heads));
  a.part_ml = w.sliced ? (float*)(at + w.ml) : nullptr;
  a.part_acc = w.sliced ? (float*)(at + w.acc) : nullptr;
  a.heads = d->kv_heads;
  a.max_len = a.max_tokens = capacity(d);
  a.num_intervals = d->num_intervals;
  a.num_splits = p.cut ? p.splits : 1;
  a.scale_log2e = scale * 1.4426950408889634f;
  a.block_table = block_table;
  a.table_pages = d->table_pages;
  a.page_shift = page_shift(d);
  a.num_pages = d->num_pages;
  a.group = d->heads / d->kv_heads;
  a.batch = d->batch;
  a.window = d->window;
  a.sinks = d->sinks;
  a.room = p.cut ? p.room : 0;
  a.more_room = p.rows;
  a.whole = paged_whole(d, fp4);
  a.least = paged_least(kind, fp4);
  a.final_ml = weights ? (float*)(at + w.final_ml) : nullptr;
  a.counts = weights && spans ? (int32_t*)(at + w.counts) : nullptr;
  a.list = weights && spans ? (int32_t*)(at + w.list) : nullptr;
  a.scores = weights ? (float*)(at + w.scores) : nullptr;
  a.weights = weights;
  a.selected = selected;
  a.budget = d->budget;
  a.weights_here = weights && p.own_weights ? 1 : 0;
  return SPAN_OK;
}

}  // namespace spanattn
#endif
