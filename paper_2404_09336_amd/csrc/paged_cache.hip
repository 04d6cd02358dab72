// What happens to the rows of a cache in pages between the attention calls: new rows go in (append), the least attended go out (evict).
// Both are copies, bound by memory, and for the few rows of a decode step by their chain of trips to it.
#include "paged_device.h"

namespace spanattn {

namespace {

// ---- append ------------------------------------------------------------------------------------------------
struct AppendArgs {
  const u32x4* k_new;
  const u32x4* v_new;
  u32x4* k;
  u32x4* v;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* q_offsets;  // or null: row b is sequence b's
  int32_t* positions;        // or null
  const int32_t* seen;       // or null
  int32_t batch, kv_heads, table_pages, page_shift, num_pages, num_tokens, max_len;
  int32_t row_pieces;        // 16-byte pieces of a row: a power of two
  int32_t chunks;            // waves per token
};

constexpr int kAppendLoads = 4;  // pieces of K and of V per lane: a wave moves up to 4 KB of each

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

// A wave takes 4 KB of one token's rows.  The rows themselves are asked for first; meanwhile the sequence is found and its page.
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t unit = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4u + (threadIdx.x >> 6)));
  const int t = (int)(unit / (uint32_t)a.chunks), c = (int)(unit % (uint32_t)a.chunks);
  if (t >= a.num_tokens) return;
  const int pieces = a.kv_heads * a.row_pieces;  // of a token
  const int first = c * 64 * kAppendLoads + lane;
  u32x4 kx[kAppendLoads], vx[kAppendLoads];
#pragma unroll
  for (int i = 0; i < kAppendLoads; ++i) {
    const int at = min(first + 64 * i, pieces - 1);
    kx[i] = __builtin_nontemporal_load(a.k_new + (size_t)t * pieces + at);
    vx[i] = __builtin_nontemporal_load(a.v_new + (size_t)t * pieces + at);
  }
  int b = t, end = t + 1;
  if (a.q_offsets != nullptr) {
    b = sequence_of(a.q_offsets, a.batch, t, lane);
    if (b < 0 || a.q_offsets[b] > t) return;
    end = a.q_offsets[b + 1];
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int len = clampi(a.ctx_lens[b], 0, a.max_len);
  const int p = __builtin_amdgcn_readfirstlane(len - end + t);
  if (p < 0) return;
  if (a.positions != nullptr && c == 0) {
    const int position = (a.seen != nullptr ? a.seen[b] : len) - end + t;
    for (int h = lane; h < a.kv_heads; h += 64) a.positions[((size_t)b * a.kv_heads + h) * (size_t)a.max_len + p] = position;
  }
  const int x = __builtin_amdgcn_readfirstlane(pool_row(a.block_table + (size_t)b * a.table_pages, p, a.page_shift, a.num_pages));
  if (x < 0) return;
  const size_t page = (size_t)(x >> a.page_shift), in_page = (size_t)(x & ((1 << a.page_shift) - 1));
#pragma unroll
  for (int i = 0; i < kAppendLoads; ++i) {
    const int at = first + 64 * i;
    if (at < pieces) {
      const int h = at / a.row_pieces, piece = at % a.row_pieces;
      const size_t to = (((page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) + in_page) * (size_t)a.row_pieces + (size_t)piece;
      a.k[to] = kx[i];
      a.v[to] = vx[i];
    }
  }
}

// ---- evict -------------------------------------------------------------------------------------------------
struct EvictArgs {
  u32x4* k;
  u32x4* v;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const float* weights;
  const int32_t* positions;
  float* weights_out;
  int32_t* positions_out;
  int32_t* new_lens;
  int32_t* moves;  // per (sequence, KV head): count, `most` slots to move to, `most` to move from
  int32_t kv_heads, table_pages, page_shift, num_pages, max_len, budget, sinks, recent, most;
};

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// Which rows stay, one workgroup per (sequence, KV head).  Every slot has a 32-bit key that orders as it is to be kept: largest for the protected ones, then the weight's
// bits made monotone; equal keys by slot.  The budget-th largest key is found two bits at a time, counting with ballots the keys that reach the three candidates of
// a step (a histogram's atomics would meet in few bins: weights share their exponents); then the waves, each with its own run of slots, count
// equal keys, free slots and rows to move, and write the lists in order.  Keys of up to kKeys slots stay in LDS, those of longer caches are made
// again from the weights each time.
template <int kKeys>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const EvictArgs a) {
  __shared__ uint32_t s_key[kKeys];
  __shared__ int s_sum[3][4];
  __shared__ int s_wave[3][kSelectWaves];
  __shared__ int s_last[kSelectWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x, b = bh / a.kv_heads;
  const int n = clampi(a.ctx_lens[b], 0, a.max_len), keep = a.budget;
  const size_t row = (size_t)bh * (size_t)a.max_len;
  const float* weights = a.weights + row;
  const int32_t* positions = a.positions != nullptr ? a.positions + row : nullptr;
  float* weights_out = a.weights_out + row;
  int32_t* positions_out = a.positions_out != nullptr ? a.positions_out + row : nullptr;
  int32_t* moves = a.moves + (size_t)bh * (size_t)(1 + 2 * a.most);
  if (n <= keep) {
    if (tid == 0) moves[0] = 0;
    for (int i = tid; i < n; i += kSelectThreads) {
      weights_out[i] = weights[i];
      if (positions_out != nullptr) positions_out[i] = positions[i];
    }
    return;
  }
  // the largest position held
  int last = n - 1;
  if (positions != nullptr) {
    last = 0;
    for (int i = tid; i < n; i += kSelectThreads) last = max(last, positions[i]);
    last = __builtin_amdgcn_readlane(wave_inclusive_max(last), 63);
    if (lane == 0) s_last[wave] = last;
    __syncthreads();
    last = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) last = max(last, s_last[w]);
  }
  auto make_key = [&](int i) -> uint32_t {
    const int p = positions != nullptr ? positions[i] : i;
    if (p < a.sinks || last - p < a.recent) return 0xffffffffu;
    const uint32_t u = __builtin_bit_cast(uint32_t, weights[i]);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;  // NaN
    if (u == 0x80000000u) return 0x80000000u;        // -0 is 0
    return u ^ ((u >> 31) != 0 ? 0xffffffffu : 0x80000000u);
  };
  const bool held = n <= kKeys;
  if (held) {
    for (int i = tid; i < n; i += kSelectThreads) s_key[i] = make_key(i);
  }
  if (tid < 12) s_sum[tid / 4][tid % 4] = 0;
  __syncthreads();
  auto key = [&](int i) -> uint32_t { return held ? s_key[i] : make_key(i); };

  uint32_t at = 0;  // the largest key that `keep` keys reach, as far as it is known
  int round = 0;
  for (int shift = 30; shift >= 0; shift -= 2, round = round == 2 ? 0 : round + 1) {
    int reach[3] = {0, 0, 0};
    for (int i0 = wave * 64; i0 < n; i0 += kSelectThreads) {
      const int i = i0 + lane;
      const uint32_t x = i < n ? key(i) : 0u;
#pragma unroll
      for (int k = 0; k < 3; ++k) reach[k] += __popcll(__builtin_amdgcn_ballot_w64(i < n && x >= at + ((uint32_t)(k + 1) << shift)));
    }
    const int next = round == 2 ? 0 : round + 1;
    if (tid < 4) s_sum[next][tid] = 0;  // (last read two barriers ago)
    if (lane < 3) atomicAdd(&s_sum[round][lane], lane == 0 ? reach[0] : (lane == 1 ? reach[1] : reach[2]));
    __syncthreads();
    const int c1 = s_sum[round][0], c2 = s_sum[round][1], c3 = s_sum[round][2];
    at += (uint32_t)(c3 >= keep ? 3 : (c2 >= keep ? 2 : (c1 >= keep ? 1 : 0))) << shift;
  }

  // waves' runs of slots
  const int run = ((n + 63) / 64 + kSelectWaves - 1) / kSelectWaves * 64;
  const int begin = min(wave * run, n), end = min(begin + run, n);
  auto lanes_below = [&](uint64_t who) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u)); };
  int above = 0, equal = 0;
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    const uint32_t x = i < end ? key(i) : 0u;
    above += __popcll(__builtin_amdgcn_ballot_w64(i < end && x > at));
    equal += __popcll(__builtin_amdgcn_ballot_w64(i < end && x == at));
  }
  if (lane == 0) {
    s_wave[0][wave] = above;
    s_wave[1][wave] = equal;
  }
  __syncthreads();
  int ties = keep, ties_before = 0;  // of the slots with key `at` so many stay: the first
  for (int w = 0; w < kSelectWaves; ++w) {
    ties -= s_wave[0][w];
    ties_before += w < wave ? s_wave[1][w] : 0;
  }
  __syncthreads();
  // pass 0 counts the wave's free slots below the budget and the rows it has to move, pass 1 writes them down
  int free_before = 0, move_before = 0, count = 0;
  for (int pass = 0; pass < 2; ++pass) {
    int tied = ties_before, holes = free_before, movers = move_before;
    for (int i0 = begin; i0 < end; i0 += 64) {
      const int i = i0 + lane;
      const bool in = i < end;
      const uint32_t x = in ? key(i) : 0u;
      const uint64_t eq = __builtin_amdgcn_ballot_w64(in && x == at);
      const bool stays = in && (x > at || (x == at && tied + lanes_below(eq) < ties));
      tied += __popcll(eq);
      const bool hole = in && !stays && i < keep, mover = stays && i >= keep;
      const uint64_t hole_lanes = __builtin_amdgcn_ballot_w64(hole), mover_lanes = __builtin_amdgcn_ballot_w64(mover);
      if (pass == 1) {
        if (hole) moves[1 + holes + lanes_below(hole_lanes)] = i;
        if (mover) moves[1 + a.most + movers + lanes_below(mover_lanes)] = i;
        if (stays && i < keep) {
          weights_out[i] = weights[i];
          if (positions_out != nullptr) positions_out[i] = positions[i];
        }
      }
      holes += __popcll(hole_lanes);
      movers += __popcll(mover_lanes);
    }
    if (pass == 0) {
      if (lane == 0) {
        s_wave[0][wave] = holes;
        s_wave[1][wave] = movers;
      }
      __syncthreads();
      for (int w = 0; w < kSelectWaves; ++w) {
        free_before += w < wave ? s_wave[0][w] : 0;
        move_before += w < wave ? s_wave[1][w] : 0;
        count += s_wave[1][w];
      }
    }
  }
  if (tid == 0) moves[0] = count;
  __syncthreads();  // the lists are written
  for (int m = tid; m < count; m += kSelectThreads) {
    const int to = moves[1 + m], from = moves[1 + a.most + m];
    weights_out[to] = weights[from];
    if (positions_out != nullptr) positions_out[to] = positions[from];
  }
  __syncthreads();  // (the outputs may be the arrays themselves)
  for (int i = keep + tid; i < n; i += kSelectThreads) {
    weights_out[i] = 0.f;
    if (positions_out != nullptr) positions_out[i] = -1;
  }
}

// The rows that move: slots from the budget on are only read, slots below it that fell free only written.
template <int kRowBytes>
__global__ __launch_bounds__(256) void move_kernel(const EvictArgs a) {
  constexpr int kLanes = kRowBytes / 16, kRows = 256 / kLanes;  // lanes of a row, rows of a workgroup at a time
  const int bh = blockIdx.x, b = bh / a.kv_heads, h = bh % a.kv_heads;
  const int32_t* moves = a.moves + (size_t)bh * (size_t)(1 + 2 * a.most);
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.new_lens[b] = min(clampi(a.ctx_lens[b], 0, a.max_len), a.budget);
  const int count = moves[0], piece = (int)threadIdx.x % kLanes;
  auto place = [&](int x) {
    const size_t page = (size_t)(x >> a.page_shift), in_page = (size_t)(x & ((1 << a.page_shift) - 1));
    return (((page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) + in_page) * (size_t)kLanes + (size_t)piece;
  };
  for (int m = (int)blockIdx.y * kRows + (int)threadIdx.x / kLanes; m < count; m += (int)gridDim.y * kRows) {
    const int to = pool_row(table, moves[1 + m], a.page_shift, a.num_pages);
    const int from = pool_row(table, moves[1 + a.most + m], a.page_shift, a.num_pages);
    if (to < 0 || from < 0) continue;
    const size_t src = place(from), dst = place(to);
    const u32x4 kx = __builtin_nontemporal_load(a.k + src), vx = __builtin_nontemporal_load(a.v + src);
    a.k[dst] = kx;
    a.v[dst] = vx;
  }
}

constexpr int64_t kMoveWorkgroups = 2048;

}  // namespace
}  // namespace spanattn

extern "C" int paged_append(const span_paged_desc_t* desc, const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                            const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, int32_t* positions,
                            const int32_t* seen) {
  using namespace spanattn;
  const int rc = check_paged(desc);
  if (rc != SPAN_OK) return rc;
  if (!q_offsets && desc->num_tokens != desc->batch) return SPAN_ERR_SHAPE;
  if (desc->num_tokens == 0) return SPAN_OK;
  if (!k_new || !v_new || !k_pages || !v_pages || !block_table || !ctx_lens) return SPAN_ERR_NULL;
  AppendArgs a;
  a.k_new = (const u32x4*)k_new;
  a.v_new = (const u32x4*)v_new;
  a.k = (u32x4*)k_pages;
  a.v = (u32x4*)v_pages;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.q_offsets = q_offsets;
  a.positions = positions;
  a.seen = seen;
  a.batch = desc->batch;
  a.kv_heads = desc->kv_heads;
  a.table_pages = desc->table_pages;
  a.page_shift = page_shift(desc);
  a.num_pages = desc->num_pages;
  a.num_tokens = desc->num_tokens;
  a.max_len = capacity(desc);
  a.row_pieces = desc->head_dim * (desc->dtype == SPAN_F32 ? 4 : 2) / 16;
  a.chunks = (desc->kv_heads * a.row_pieces + 64 * kAppendLoads - 1) / (64 * kAppendLoads);
  const int64_t units = (int64_t)desc->num_tokens * a.chunks;
  if (units > INT32_MAX) return SPAN_ERR_SHAPE;
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, (hipStream_t)desc->stream, a);
  return launched();
}

extern "C" int paged_evict(const span_paged_desc_t* desc, void* k_pages, void* v_pages, const int32_t* block_table, const int32_t* ctx_lens,
                           const float* weights, const int32_t* positions, float* weights_out, int32_t* positions_out, int32_t* new_lens) {
  using namespace spanattn;
  const int rc = check_paged(desc);
  if (rc != SPAN_OK) return rc;
  if (desc->budget <= 0 || (int64_t)desc->sinks + desc->recent > desc->budget) return SPAN_ERR_SHAPE;
  if (!k_pages || !v_pages || !block_table || !ctx_lens || !weights || !weights_out || !new_lens) return SPAN_ERR_NULL;
  if ((positions == nullptr) != (positions_out == nullptr)) return SPAN_ERR_NULL;
  if (!desc->workspace || ((uintptr_t)desc->workspace & 255u) || desc->workspace_bytes < evict_workspace(desc)) return SPAN_ERR_WORKSPACE;
  EvictArgs a;
  a.k = (u32x4*)k_pages;
  a.v = (u32x4*)v_pages;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.weights = weights;
  a.positions = positions;
  a.weights_out = weights_out;
  a.positions_out = positions_out;
  a.new_lens = new_lens;
  a.moves = (int32_t*)desc->workspace;
  a.kv_heads = desc->kv_heads;
  a.table_pages = desc->table_pages;
  a.page_shift = page_shift(desc);
  a.num_pages = desc->num_pages;
  a.max_len = capacity(desc);
  a.budget = desc->budget;
  a.sinks = desc->sinks;
  a.recent = desc->recent;
  a.most = a.max_len > a.budget ? (a.max_len - a.budget < a.budget ? a.max_len - a.budget : a.budget) : 0;
  const unsigned pairs = (unsigned)desc->batch * (unsigned)desc->kv_heads;
  hipStream_t stream = (hipStream_t)desc->stream;
  constexpr int kSmall = 8192, kLarge = 32768;
  if (a.max_len <= kSmall) hipLaunchKernelGGL(select_kernel<kSmall>, dim3(pairs), dim3(kSelectThreads), 0, stream, a);
  else hipLaunchKernelGGL(select_kernel<kLarge>, dim3(pairs), dim3(kSelectThreads), 0, stream, a);
  const int src = launched();
  if (src != SPAN_OK) return src;
  const int row_bytes = desc->head_dim * (desc->dtype == SPAN_F32 ? 4 : 2), rows = 256 / (row_bytes / 16);
  int64_t splits = (kMoveWorkgroups + pairs - 1) / pairs;
  const int64_t useful = (a.most + rows - 1) / rows;
  if (splits > useful) splits = useful;
  if (splits < 1) splits = 1;
  const dim3 grid(pairs, (unsigned)splits);
  if (row_bytes == 128) hipLaunchKernelGGL(move_kernel<128>, grid, dim3(256), 0, stream, a);
  else if (row_bytes == 256) hipLaunchKernelGGL(move_kernel<256>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(move_kernel<512>, grid, dim3(256), 0, stream, a);
  return launched();
}
