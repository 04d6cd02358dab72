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

// A wave takes 4 KB of one token's rows.  The rows themselves are asked for first; meanwhile the sequence is found and its page.  Prompts of 16 sequences
// (20600 rows of 32 heads of 128, bf16) take 126 us, 5.35 TB/s read and written, which is what a large copy reaches; 64 rows of a step 3.4 us, a launch's least.
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
  const int len = a.ctx_lens[b];
  const int p = __builtin_amdgcn_readfirstlane((int)((uint32_t)len - (uint32_t)end + (uint32_t)t));
  if ((uint32_t)p >= (uint32_t)a.max_len) return;  // no place in the table: ahead of its first position, or the table is full
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
  uint32_t* counters;  // tickets: of every (sequence, KV head), then of every sequence; zero between calls
  int32_t* moves;      // per (sequence, KV head): count, 0, `most` pairs of slots, to and from
  int32_t kv_heads, table_pages, page_shift, num_pages, max_len, budget, sinks, recent, most, row_shift, in_place;
};

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kHoleList = 4096;  // free slots whose list fits LDS

// A pair's rows that move, pair_of(m) = (to, from) for m < count, by `threads` threads.  Slots from the budget on are only read, slots below it that fell
// free only written, so the order does not matter.
template <class PairOf>
static __device__ __forceinline__ void move_rows(const EvictArgs& a, int bh, int thread, int threads, int count, PairOf&& pair_of) {
  const int b = bh / a.kv_heads, h = bh % a.kv_heads;
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;
  const int piece = thread & ((1 << a.row_shift) - 1), rows = threads >> a.row_shift;
  auto place = [&](int x) {
    const size_t page = (size_t)(x >> a.page_shift), in_page = (size_t)(x & ((1 << a.page_shift) - 1));
    return (((((page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) + in_page)) << a.row_shift) + (size_t)piece;
  };
  constexpr int kAhead = 2;  // rows of a thread on their way
  for (int m0 = thread >> a.row_shift; m0 < count; m0 += kAhead * rows) {
    int to[kAhead], from[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int m = m0 + k * rows;
      const i32x2 pair = pair_of(min(m, count - 1));
      to[k] = pool_row(table, pair[0], a.page_shift, a.num_pages);
      from[k] = pool_row(table, pair[1], a.page_shift, a.num_pages);
      if (m >= count || from[k] < 0) to[k] = -1;
    }
    u32x4 kx[kAhead], vx[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      kx[k] = __builtin_nontemporal_load(a.k + place(max(from[k], 0)));  // (some row of the pool rather than a branch)
      vx[k] = __builtin_nontemporal_load(a.v + place(max(from[k], 0)));
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (to[k] >= 0) {
        a.k[place(to[k])] = kx[k];
        a.v[place(to[k])] = vx[k];
      }
    }
  }
}

// Which rows stay, one workgroup per (sequence, KV head).  Every slot has a 32-bit key that orders as it is to be kept: largest for the protected ones, then the
// weight's bits made monotone, 1 for NaN, 0 for no slot; equal keys by slot.  The budget-th largest key is found digit by digit (11, 11 and 10 bits) with histograms in LDS; the
// first digit holds a weight's exponent and two bits of its mantissa, so that even weights of one size spread over some bins, and the protected ones, which
// all meet, are counted apart.  Then the waves, each with its own run of slots, count equal keys, free slots and rows to move in order.
// kKeys: slots of a thread, whose keys stay in registers; 0: any number, keys made again from the weights each time.
// With keys in registers the workgroup also moves rows: where the card has more CUs than there are pairs, each pair has several workgroups that find the
// same selection and move a part of the rows each, so nothing waits for a second launch.  Longer caches leave the list in the workspace, for move_kernel.
// What bounds it: the passes over a CU's slots are bound by instructions (some 15 a piece of 64 slots in each of seven passes), the moves by memory.
// us of a call, 16 x 8 caches of ~4350 slots down to 4096 and 5 x 16 of 900 .. 12000 down to 2048: keys in LDS and two bits a step by ballots, and a second
// launch that moves: 40 and 75; histograms of three digits, keys in registers: 23.3 and 32.3; one launch, fewer instructions a piece: 18.0 and 27.5.
// (With outputs in place, whose writers are found by tickets, a call of few rows takes about 1 us more.)
template <int kKeys>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(const EvictArgs a) {
  constexpr bool kMoves = kKeys > 0;
  __shared__ int s_bins[2048];
  __shared__ int s_holes[kMoves ? 1 : kHoleList];
  __shared__ uint16_t s_pairs[kMoves ? kKeys * kSelectThreads / 2 : 1][2];  // to and from (half of the slots at most: one falls free for each that moves)
  __shared__ int s_wave[6][kSelectWaves];  // (a row of its own for all that no barrier parts)
  __shared__ int s_pick[3];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x, b = bh / a.kv_heads;
  const int n = clampi(a.ctx_lens[b], 0, a.max_len), keep = a.budget;
  const int part = kMoves ? (int)blockIdx.y : 0, parts = kMoves ? (int)gridDim.y : 1;
  const size_t row = (size_t)bh * (size_t)a.max_len;
  const float* weights = a.weights + row;
  const int32_t* positions = a.positions != nullptr ? a.positions + row : nullptr;
  float* weights_out = a.weights_out + row;
  int32_t* positions_out = a.positions_out != nullptr ? a.positions_out + row : nullptr;
  int32_t* moves = a.moves + (size_t)bh * (size_t)(2 + 2 * a.most);
  if (n <= keep) {
    if (kMoves && bh % a.kv_heads == 0 && part == 0 && tid == 0) a.new_lens[b] = n;  // (which is what others may still read there)
    if (!kMoves && tid == 0) moves[0] = 0;
    for (int i = part * kSelectThreads + tid; i < n; i += parts * kSelectThreads) {
      weights_out[i] = weights[i];
      if (positions_out != nullptr) positions_out[i] = positions[i];
    }
    return;
  }
  // the wave's run of slots, in pieces of 64
  const int run = ((n + 63) / 64 + kSelectWaves - 1) / kSelectWaves * 64;
  const int begin = min(wave * run, n), end = min(begin + run, n);
  auto pieces = [&](auto&& f) {
    if constexpr (kKeys > 0) {
#pragma unroll
      for (int j = 0; j < kKeys; ++j) {
        if (begin + 64 * j < end) f(j, begin + 64 * j + lane);
      }
    } else {
      for (int i0 = begin; i0 < end; i0 += 64) f(0, i0 + lane);
    }
  };
  constexpr int kHeld = kKeys > 0 ? kKeys : 1;
  constexpr bool kRemember = kKeys > 0 && kKeys <= 16;  // weights and positions too (32 of each would spill)
  uint32_t held[kHeld];  // keys
  float weight[kHeld];
  // the weights, and the largest position held
  int last = n - 1;
  if constexpr (kKeys > 0) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) weight[j] = begin + 64 * j < end ? weights[min(begin + 64 * j + lane, n - 1)] : 0.f;
  }
  int position[kHeld];
  if (positions != nullptr) {
    last = 0;
    if constexpr (kKeys > 0) {
#pragma unroll
      for (int j = 0; j < kKeys; ++j) position[j] = begin + 64 * j < end ? positions[min(begin + 64 * j + lane, n - 1)] : 0;
#pragma unroll
      for (int j = 0; j < kKeys; ++j) last = max(last, position[j]);
    } else {
      for (int i = tid; i < n; i += kSelectThreads) last = max(last, positions[i]);
    }
    last = __builtin_amdgcn_readlane(wave_inclusive_max(last), 63);
    if (lane == 0) s_wave[3][wave] = last;
  }
  i32x2& bins = *reinterpret_cast<i32x2*>(&s_bins[2 * tid]);
  bins = i32x2{0, 0};
  __syncthreads();
  auto over_waves = [&](int which) { return lane < kSelectWaves ? s_wave[which][lane] : 0; };  // (summed or scanned by every wave for itself)
  if (positions != nullptr) last = __builtin_amdgcn_readlane(wave_inclusive_max(over_waves(3)), 63);
  auto key_of = [&](int p, uint32_t u) -> uint32_t {
    if (p < a.sinks || last - p < a.recent) return 0xffffffffu;
    if ((u & 0x7fffffffu) > 0x7f800000u) return 1u;  // NaN
    if (u == 0x80000000u) return 0x80000000u;        // -0 is 0
    return u ^ ((u >> 31) != 0 ? 0xffffffffu : 0x80000000u);
  };
  if constexpr (kKeys > 0) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const int i = begin + 64 * j + lane;
      held[j] = i < end ? key_of(positions != nullptr ? position[j] : i, __builtin_bit_cast(uint32_t, weight[j])) : 0u;
    }
  }
  auto key = [&](int j, int i) -> uint32_t {
    if constexpr (kKeys > 0) return held[j];
    else return i < end ? key_of(positions != nullptr ? positions[i] : i, __builtin_bit_cast(uint32_t, weights[i])) : 0u;
  };
  auto count_if = [&](bool x) { return (int)__popcll(__builtin_amdgcn_ballot_w64(x)); };
  auto lanes_below = [&](uint64_t who) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u)); };

  int safe = 0;
  pieces([&](int j, int i) {
    const uint32_t x = key(j, i);
    safe += count_if(x == 0xffffffffu);
    if (x != 0xffffffffu) atomicAdd(&s_bins[2047 - (int)(x >> 21)], 1);
  });
  if (lane == 0) s_wave[0][wave] = safe;
  __syncthreads();
  // All of the workgroup's threads hold their weights and positions now.  Where outputs are inputs, the last of a pair's workgroups to come here writes all of
  // the pair's, and the last of a sequence's the length.  (Nothing that others write is read after it, and these reads are done: no ordering is needed.)
  uint32_t ticket = 0, sequence_ticket = 0;
  if (kMoves && a.in_place != 0 && tid == 0) {
    if (parts > 1) ticket = __hip_atomic_fetch_add(a.counters + bh, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sequence_ticket = __hip_atomic_fetch_add(a.counters + gridDim.x + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  safe = __builtin_amdgcn_readlane(wave_inclusive_scan(over_waves(0)), 63);
  uint32_t at = 0xffffffffu;  // the key of the last row that stays
  int ties = keep;            // of the slots with that key so many stay, the first
  int tied_slots = safe;      // the slots with that key
  if (safe < keep) {
    ties = keep - safe;
    at = 0;
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {  // (bins count from the largest)
      const int shift = digit == 0 ? 21 : (digit == 1 ? 10 : 0);
      if (digit > 0) {
        const int above = digit == 1 ? 21 : 10, mask = digit == 1 ? 2047 : 1023;
        pieces([&](int j, int i) {
          const uint32_t x = key(j, i);
          if (x != 0xffffffffu && (x ^ at) >> above == 0) atomicAdd(&s_bins[mask - (int)(x >> shift & (uint32_t)mask)], 1);
        });
        __syncthreads();
      }
      const int c0 = bins[0], c1 = bins[1];
      const int incl = wave_inclusive_scan(c0 + c1);
      if (lane == 63) s_wave[1][wave] = incl;
      __syncthreads();
      bins = i32x2{0, 0};
      const int waves_incl = wave_inclusive_scan(over_waves(1));
      const int before = incl - c0 - c1 + (wave > 0 ? __builtin_amdgcn_readlane(waves_incl, wave - 1) : 0);
      if (before < ties && before + c0 + c1 >= ties) {
        const bool first = before + c0 >= ties;
        s_pick[0] = 2 * tid + (first ? 0 : 1);
        s_pick[1] = before + (first ? 0 : c0);
        s_pick[2] = first ? c0 : c1;
      }
      __syncthreads();
      at |= (uint32_t)((digit == 2 ? 1023 : 2047) - s_pick[0]) << shift;
      ties -= s_pick[1];
      tied_slots = s_pick[2];
    }
  }

  auto before_wave = [&](int which) {
    const int incl = wave_inclusive_scan(over_waves(which));
    return wave > 0 ? __builtin_amdgcn_readlane(incl, wave - 1) : 0;
  };
  const bool all_tied = ties == tied_slots;  // (the common case: weights differ)
  int ties_before = 0;
  if (!all_tied) {
    int equal = 0;
    pieces([&](int j, int i) { equal += count_if(key(j, i) == at); });
    if (lane == 0) s_wave[2][wave] = equal;
    __syncthreads();
    ties_before = before_wave(2);
  }
  int tied = ties_before;
  auto who_stays = [&](int j, int i) -> uint64_t {  // called piece by piece
    const uint32_t x = key(j, i);
    if (all_tied) return __builtin_amdgcn_ballot_w64(x >= at);
    const uint64_t eq = __builtin_amdgcn_ballot_w64(x == at);
    const bool yes = x > at || (x == at && tied + lanes_below(eq) < ties);
    tied += __popcll(eq);
    return __builtin_amdgcn_ballot_w64(yes);
  };
  // of a piece: the slots below the budget that fall free, the rows beyond it that stay
  const int below = min(end, keep);
  auto free_slots = [&](uint64_t stay, int i) { return ~stay & __builtin_amdgcn_ballot_w64(i < below); };
  auto moving = [&](uint64_t stay, int i) { return stay & __builtin_amdgcn_ballot_w64(i >= keep); };
  int holes = 0, movers = 0;
  uint64_t staying[kHeld];  // registers: found once
  pieces([&](int j, int i) {
    const uint64_t stay = who_stays(j, i);
    if constexpr (kKeys > 0) staying[j] = stay;
    holes += __popcll(free_slots(stay, i));
    movers += __popcll(moving(stay, i));
  });
  if (lane == 0) {
    s_wave[4][wave] = holes;
    s_wave[5][wave] = movers;
  }
  if (kMoves && tid == 0) s_last = ticket == (uint32_t)(parts - 1) ? 1 : 0;
  __syncthreads();
  holes = before_wave(4);
  movers = before_wave(5);
  const int num_moves = __builtin_amdgcn_readlane(wave_inclusive_scan(over_waves(5)), 63);
  // The free slots are listed; then who moves reads its slot, writes the pair down and its weight and position there.  Every slot's own weight and
  // position are read by its own thread only, ahead of what it writes, so the outputs may be the arrays themselves: a free slot's are not needed.
  const bool in_lds = kMoves || num_moves <= kHoleList;
  tied = ties_before;
  int at_hole = holes, at_mover = movers;
  pieces([&](int j, int i) {
    uint64_t stay;
    if constexpr (kKeys > 0) stay = staying[j];
    else stay = who_stays(j, i);
    const uint64_t who = free_slots(stay, i);
    if (who != 0) {
      const int m = at_hole + lanes_below(who);
      if (who >> lane & 1u) {
        if constexpr (kMoves) s_pairs[m][0] = (uint16_t)i;
        else (in_lds ? s_holes[m] : moves[2 + 2 * m]) = i;
      }
      at_hole += __popcll(who);
    }
    if constexpr (kMoves) {
      const uint64_t from = moving(stay, i);
      if (from != 0) {
        if (from >> lane & 1u) s_pairs[at_mover + lanes_below(from)][1] = (uint16_t)i;
        at_mover += __popcll(from);
      }
    }
  });
  __syncthreads();
  if constexpr (kMoves) {
    move_rows(a, bh, part * kSelectThreads + tid, parts * kSelectThreads, num_moves, [&](int m) {
      const uint32_t pair = *reinterpret_cast<const uint32_t*>(s_pairs[m]);
      return i32x2{(int)(pair & 0xffffu), (int)(pair >> 16)};
    });
    if (tid == 0) {
      if (a.in_place == 0) {
        if (bh % a.kv_heads == 0 && part == 0) a.new_lens[b] = keep;
      } else if (sequence_ticket == (uint32_t)(a.kv_heads * parts - 1)) {
        __hip_atomic_store(a.counters + gridDim.x + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        a.new_lens[b] = keep;
      }
    }
    if (a.in_place != 0 && parts > 1) {
      if (s_last == 0) return;
      if (tid == 0) __hip_atomic_store(a.counters + bh, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  } else if (tid == 0) {
    moves[0] = num_moves;
  }
  tied = ties_before;
  at_mover = movers;
  pieces([&](int j, int i) {
    uint64_t stay;
    if constexpr (kKeys > 0) stay = staying[j];
    else stay = who_stays(j, i);
    const uint64_t who = moving(stay, i);
    const int m = at_mover + lanes_below(who);
    at_mover += __popcll(who);
    if (kMoves && a.in_place == 0 && (uint32_t)(i - lane) / 64u % (uint32_t)parts != (uint32_t)part) return;  // (another workgroup's)
    const bool yes = stay >> lane & 1u, mover = who >> lane & 1u;
    if (i < end) {
      float w = 0.f;
      int p = -1;
      if (yes) {
        if constexpr (kRemember) {
          w = weight[j];
          if (positions != nullptr) p = position[j];
        } else {
          w = weights[i];
          if (positions != nullptr) p = positions[i];
        }
      }
      if (mover) {
        int to;
        if constexpr (kMoves) {
          to = s_pairs[m][0];
        } else {
          to = in_lds ? s_holes[m] : moves[2 + 2 * m];
          *reinterpret_cast<i32x2*>(moves + 2 + 2 * m) = i32x2{to, i};
        }
        if (kKeys > 0) {
          weights_out[to] = w;
          if (positions_out != nullptr) positions_out[to] = p;
        }
      }
      if (kKeys > 0 || i < keep) {
        if (i >= keep || yes) {
          weights_out[i] = i < keep ? w : 0.f;
          if (positions_out != nullptr) positions_out[i] = i < keep ? p : -1;
        }
      }
    }
  });
  if constexpr (kKeys == 0) {
    // (keys were made from the arrays up to here: what changes a weight or a position that a key is made from comes after them all)
    __syncthreads();
    for (int m = tid; m < num_moves; m += kSelectThreads) {
      const int to = moves[2 + 2 * m], from = moves[3 + 2 * m];
      weights_out[to] = weights[from];
      if (positions_out != nullptr) positions_out[to] = positions[from];
    }
    __syncthreads();
    for (int i = keep + tid; i < n; i += kSelectThreads) {
      weights_out[i] = 0.f;
      if (positions_out != nullptr) positions_out[i] = -1;
    }
  }
}

// The rows that move, of lists that select_kernel left in the workspace.
__global__ __launch_bounds__(256) void move_kernel(const EvictArgs a) {
  const int bh = blockIdx.x, b = bh / a.kv_heads;
  const int32_t* moves = a.moves + (size_t)bh * (size_t)(2 + 2 * a.most);
  if (bh % a.kv_heads == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.new_lens[b] = min(clampi(a.ctx_lens[b], 0, a.max_len), a.budget);
  move_rows(a, bh, (int)(blockIdx.y * 256 + threadIdx.x), (int)gridDim.y * 256, moves[0],
            [&](int m) { return *reinterpret_cast<const i32x2*>(moves + 2 + 2 * m); });
}

constexpr int64_t kMoveWorkgroups = 2048;
// A pair gets several workgroups while there are CUs for them and rows for one pass of each.  The batch of 16 x 8 caches above takes 20 us with 256 workgroups
// and 30 with 512, whose second halves select once more when the first are done; rows for one, two and four passes: 12.3, 13.8 and 17.8 us for 2 x 32 caches of
// 1700 slots.
constexpr unsigned kSelectWorkgroups = 256;

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
  a.counters = (uint32_t*)desc->workspace;
  a.moves = (int32_t*)((char*)desc->workspace + counter_bytes(desc));
  a.kv_heads = desc->kv_heads;
  a.table_pages = desc->table_pages;
  a.page_shift = page_shift(desc);
  a.num_pages = desc->num_pages;
  a.max_len = capacity(desc);
  a.budget = desc->budget;
  a.sinks = desc->sinks;
  a.recent = desc->recent;
  a.most = most_moves(desc);
  const unsigned pairs = (unsigned)desc->batch * (unsigned)desc->kv_heads;
  const int row_bytes = desc->head_dim * (desc->dtype == SPAN_F32 ? 4 : 2);
  a.row_shift = 31 - __builtin_clz((unsigned)row_bytes / 16u);
  hipStream_t stream = (hipStream_t)desc->stream;
  const unsigned passes = (unsigned)a.most / (unsigned)(kSelectThreads >> a.row_shift);
  const unsigned parts = std::max(std::min(kSelectWorkgroups / pairs, passes), 1u);
  const size_t slots = (size_t)pairs * (size_t)a.max_len * 4, lens = (size_t)desc->batch * 4;
  auto meet = [](const void* x, size_t x_bytes, const void* y, size_t y_bytes) {
    return x != nullptr && y != nullptr && (uintptr_t)x < (uintptr_t)y + y_bytes && (uintptr_t)y < (uintptr_t)x + x_bytes;
  };
  a.in_place = meet(ctx_lens, lens, new_lens, lens);
  for (const void* x : {(const void*)weights, (const void*)positions}) {
    for (const void* y : {(const void*)weights_out, (const void*)positions_out}) a.in_place |= meet(x, slots, y, slots);
  }
  auto select = [&](auto keys) {
    constexpr int kKeys = decltype(keys)::value;
    hipLaunchKernelGGL(select_kernel<kKeys>, dim3(pairs, kKeys > 0 ? parts : 1), dim3(kSelectThreads), 0, stream, a);
  };
  if (a.max_len <= 2 * kSelectThreads) select(std::integral_constant<int, 2>{});
  else if (a.max_len <= 8 * kSelectThreads) select(std::integral_constant<int, 8>{});
  else if (a.max_len <= 16 * kSelectThreads) select(std::integral_constant<int, 16>{});
  else if (a.max_len <= kMostKeysHeld) select(std::integral_constant<int, 32>{});
  else select(std::integral_constant<int, 0>{});
  const int src = launched();
  if (src != SPAN_OK || a.max_len <= kMostKeysHeld) return src;
  const int rows = 256 >> a.row_shift;
  int64_t splits = (kMoveWorkgroups + pairs - 1) / pairs;
  const int64_t useful = (a.most + rows - 1) / rows;
  if (splits > useful) splits = useful;
  if (splits < 1) splits = 1;
  hipLaunchKernelGGL(move_kernel, dim3(pairs, (unsigned)splits), dim3(256), 0, stream, a);
  return launched();
}
