// One-token attention over a cache held in 4 bits, for up to 16 query heads per KV head.
//
// A workgroup of 4 wavefronts takes one slice of a (sequence, KV head) pair's positions and all query heads of the group, the columns of 16x16 matrix products; slices and the
// joining of states are those of the 16- and 32-bit caches (paged_attend.h).  What differs:
//   * Positions go in units of 16 aligned ones, which lie on one page: a unit's address and the mask of its rows are wave-uniform, found by the lanes 64 units at a
//     time, and every load is contiguous over the wave.  Where a window, a span or the cache begins or ends inside a unit, its other rows are masked; two intervals that meet in a unit are two units.
//   * K stays as it is: fp4 x fp6 products with both exponents applied by the matrix core.  q is laid out as kDigits digits to the base 16, each -16 .. 16 times a power of two that 32 channels share:
//     such a digit is an fp6 value (E2M3) exactly.  (The matrix core adds eight neighbouring products up with some 13 bits below the largest, measured; products of digits fit that, those of
//     floating values of different size do not.)  Five digits hold 21 bits below the largest channel of a block, six 25.
//   * V becomes bf16, exactly, times its exponent: one instruction for two values, and one for each two that brings neighbouring positions together.  Weights meet it in three bf16 terms, all 24 bits.
#include "paged_attend.h"

namespace spanattn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef const SPAN_GLOBAL uint8_t* global_u8;
typedef const SPAN_GLOBAL uint32_t* global_u32;

constexpr int kUnitRows = kFp4Rows;
constexpr int kStepUnits = 2;                  // units that a wave takes together: 32 positions of one product with V
constexpr int kStepRows = kUnitRows * kStepUnits;
constexpr int kHeldUnits = 64;                 // of a wave, found at a time: one per lane

template <class Elt>
constexpr int kDigitsOf = Elt::kBytes == 4 ? 6 : 5;

// Units of a dense call: those of the first `sinks` positions, then those from `low` on.
struct SeenUnits {
  int sinks, low, held, first;  // positions; units of the sinks
};
__device__ __forceinline__ SeenUnits seen_units(const PagedArgs& a, int len) {
  const Seen s = seen_by_last(len, a.max_len, a.window, a.sinks);
  return SeenUnits{s.sinks, s.low, clampi(len, 0, a.max_len), (s.sinks + kUnitRows - 1) / kUnitRows};
}
__device__ __forceinline__ int unit_count(const SeenUnits& s) {
  return s.first + (s.held > s.low ? (s.held + kUnitRows - 1) / kUnitRows - s.low / kUnitRows : 0);
}

// Units of an interval [start, end) of a span list: none if it is empty.
__device__ __forceinline__ int interval_units(const PagedArgs& a, int start, int end, int& from, int& to) {
  from = clampi(start, 0, a.max_len);
  to = clampi(end, from, a.max_len);
  return to > from ? (to + kUnitRows - 1) / kUnitRows - from / kUnitRows : 0;
}

// More units than any valid list of so many intervals has (those are disjoint); sums of invalid ones stop here.
__device__ __forceinline__ int most_units(const PagedArgs& a, int intervals) { return a.max_len / kUnitRows + min(intervals, a.max_len) + 1; }

// Rows [from, to) of unit u as bits.
__device__ __forceinline__ uint32_t unit_mask(int u, int from, int to) {
  const int lo = clampi(from - u * kUnitRows, 0, kUnitRows), hi = clampi(to - u * kUnitRows, 0, kUnitRows);
  return ((1u << hi) - 1u) & ~((1u << lo) - 1u);
}

template <class Elt, int D>
__device__ __forceinline__ void lay_digits(const PagedArgs& a, size_t row0, int group, uint32_t (*s_digits)[16][D / 32][6], uint8_t (*s_exps)[16][D / 32]) {
  constexpr int kDigits = kDigitsOf<Elt>, kHalves = D / 16;  // sixteen channels of one digit per thread
  for (int i = threadIdx.x; i < 16 * kHalves * kDigits; i += kThreads) {
    const int half = i % kHalves, j = i / kHalves % 16, t = i / (kHalves * 16);
    const int block = half / 2, word = half % 2 * 3;
    if (j >= group) {
      for (int w = 0; w < 3; ++w) s_digits[t][j][block][word + w] = 0u;
      s_exps[t][j][block] = 127;
      continue;
    }
    float x[16];
    const u32x4* from = (const u32x4*)((const char*)a.q + (row0 + (size_t)j) * (size_t)(D * Elt::kBytes) + (size_t)(half * 16 * Elt::kBytes));
#pragma unroll
    for (int p = 0; p < Elt::kBytes; ++p) {
      u32x4 piece = from[p];
#pragma unroll
      for (int k = 0; k < 4; ++k) piece[k] = Elt::scale_query(piece[k], a.scale_log2e);
      Elt::unpack(piece, x + p * Elt::kPerVec);
    }
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) most = max(most, __builtin_bit_cast(uint32_t, x[k]) & 0x7fffffffu);
    most = max(most, (uint32_t)dpp_i<0xB1>((int)most));  // the block's other half is the next thread's
    // |x| < 2^(e - 126), e the largest's exponent bits; digit t counts 2^(e - 126 - 4 (t + 1)), as an fp6 value 8 times that each
    const int e = max((int)(most >> 23), 1);
    const int scale = e - 126 - 4 * (t + 1) + 3 + 127;
    s_exps[t][j][block] = (uint8_t)(most >= 0x7f800000u ? 255 : max(scale, 0));  // (not finite: NaN)
    uint32_t words[3] = {0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      // what the digits ahead of this one leave: x less its nearest multiple of the last one's unit (ties fall the same way for all threads)
      const float y = ldexpf(x[k], 126 - e + 4 * t), rest = t == 0 ? y : y - rintf(y);
      const int digit = (int)rintf(rest * 16.f);
      const uint32_t code = scale < 0 ? 0u : (uint32_t)abs(digit) | (digit < 0 ? 32u : 0u);
      const int bit = 6 * k;
      words[bit / 32] |= code << (bit % 32);
      if (bit % 32 > 26) words[bit / 32 + 1] |= code >> (32 - bit % 32);
    }
    for (int w = 0; w < 3; ++w) s_digits[t][j][block][word + w] = words[w];
  }
}

template <class Elt, int D, PagedKind kKind, class Args>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3, 3))) void fp4_kernel(const Args a) {
  constexpr bool kSpans = kKind == kPagedSpans;
  constexpr int kDigits = kDigitsOf<Elt>, kBlocks = D / 32, NE = D / 16;
  constexpr uint32_t kUnitBytes = 8u * D, kUnitExps = D / 2u;
  constexpr int kAccRow = D + 4, kTerms = 3;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qi = lane & 15, c4 = lane >> 4;
  const int h = blockIdx.x, kv_heads = a.heads, group = a.group;

  struct Queries {
    uint32_t digits[kDigits][16][kBlocks][6];
    uint8_t exps[kDigits][16][kBlocks];
  };
  union Overlaid {
    Queries q;
    float acc[kWavesPerBlock][16][kAccRow];
  };
  __shared__ __attribute__((aligned(16))) Overlaid s_u;
  __shared__ __attribute__((aligned(16))) f32x2 s_ml[16][kWavesPerBlock];
  __shared__ uint32_t s_ticket;

  Slice sl;
  if constexpr (Args::kHasTable) {
    const uint32_t entry = a.table[blockIdx.y];
    sl = Slice{(int)(entry & 1023u), (int)(entry >> 10 & 2047u), (int)(entry >> 21), 0, 0};
    sl.y0 = (int)blockIdx.y - sl.split;
  } else if (!kSpans && a.room > 0) {
    sl = locate_slice(a, (int)blockIdx.y, lane, [&](int len) { return unit_count(seen_units(a, len)) * kUnitRows; });
    if (sl.b < 0) return;  // (the grid holds the most slices that any lengths give)
  } else {
    sl.nsl = a.num_splits;
    sl.b = (int)blockIdx.y / sl.nsl;
    sl.split = (int)blockIdx.y - sl.b * sl.nsl;
    sl.y0 = sl.b * sl.nsl;
  }
  const int b = sl.b;
  const size_t bh = (size_t)b * kv_heads + h;
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;
  const float post = Elt::post_scale(a.scale_log2e);  // weight = exp2((score - largest score) * post)

  lay_digits<Elt, D>(a, bh * (size_t)group, group, s_u.q.digits, s_u.q.exps);

  SeenUnits seen = {0, 0, 0, 0};
  int first_interval = 0, intervals = 0, all;  // units of the sequence
  if constexpr (kSpans) {
    const int lo = clampi(__builtin_amdgcn_readfirstlane(a.offsets[b]), 0, a.num_intervals);
    first_interval = lo;
    intervals = clampi(__builtin_amdgcn_readfirstlane(a.offsets[b + 1]), lo, a.num_intervals) - lo;
    all = 0;
    for (int i0 = 0; i0 < intervals; i0 += 64) {
      int from, to, n = 0;
      if (i0 + lane < intervals) n = interval_units(a, a.starts[lo + i0 + lane], a.ends[lo + i0 + lane], from, to);
      all = min(all + __builtin_amdgcn_readlane(wave_inclusive_scan(n), 63), most_units(a, intervals));
    }
  } else {
    if (a.room == 0) sl.len = __builtin_amdgcn_readfirstlane(a.ctx_lens[b]);
    seen = seen_units(a, sl.len);
    all = unit_count(seen);
  }
  all = __builtin_amdgcn_readfirstlane(all);
  // even shares of whole steps, which go round the waves
  const int steps_all = (all + kStepUnits - 1) / kStepUnits;
  const int share = (steps_all + sl.nsl - 1) / sl.nsl;
  const int step0 = min(sl.split * share, steps_all), step1 = min(step0 + share, steps_all);
  const int steps = step1 - step0 > wave ? (step1 - step0 - wave + kWavesPerBlock - 1) / kWavesPerBlock : 0;  // of this wave

  const size_t page_bytes = (size_t)(D / 2 + D / kFp4Block) << a.page_shift;
  const int unit_shift = a.page_shift - 4;  // log2 of a page's units
  const char* k_head = (const char*)a.k + (size_t)h * page_bytes;
  const char* v_head = (const char*)a.v + (size_t)h * page_bytes;
  const size_t page_stride = page_bytes * (size_t)kv_heads;
  const uint32_t exps_at = (uint32_t)(D / 2) << a.page_shift;

  // The wave's units from its unit w0 on, one per lane: unit of the pool (page * units of a page + unit in the page) and mask of the rows that take part.
  int held_unit = 0;
  uint32_t held_mask = 0;
  auto find_units = [&](int w0) {
    const int w = w0 + lane, s = step0 + wave + w / kStepUnits * kWavesPerBlock;
    const int v = s * kStepUnits + w % kStepUnits;  // among the sequence's units
    const bool mine = w / kStepUnits < steps && v < all;
    int u = -1;
    held_mask = 0;
    if constexpr (kSpans) {
      int before = 0;
      for (int i0 = 0; i0 < intervals; i0 += 64) {
        int from = 0, to = 0, n = 0;
        if (i0 + lane < intervals) n = interval_units(a, a.starts[first_interval + i0 + lane], a.ends[first_interval + i0 + lane], from, to);
        const int incl = wave_inclusive_scan(n);
        // the first interval whose units end behind v
        int at = 0;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) {
          if (__shfl(incl, at + step - 1) + before <= v) at += step;
        }
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int ex = __shfl(incl - n, at & 63), f = __shfl(from, at & 63), t = __shfl(to, at & 63);
        if (mine && v >= before && v < before + total) {
          u = f / kUnitRows + (v - before - ex);
          held_mask = unit_mask(u, f, t);
        }
        before = min(before + total, most_units(a, intervals));
      }
    } else {
      const bool sink = v < seen.first;
      u = sink ? v : v - seen.first + seen.low / kUnitRows;
      if (mine) held_mask = unit_mask(u, sink ? 0 : seen.low, sink ? seen.sinks : seen.held);
    }
    int x = -1;
    if (mine && held_mask != 0) x = pool_row(table, u * kUnitRows, a.page_shift, a.num_pages);
    if (x < 0) held_mask = 0;
    held_unit = max(x, 0) / kUnitRows;  // (none: the pool's first, which nobody attends)
  };

  float ref = -INFINITY, lsum = 0.f;
  f32x4 O[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e) O[e] = f32x4{0.f, 0.f, 0.f, 0.f};

  // What a lane holds of a unit.  D = 128: K of row qi, channels 32 c4 on; D = 64: of two units together, K of row qi, unit c4 / 2, channels 32 (c4 % 2) on.  V of rows 4 c4 .. + 3, channels NE qi on.
  constexpr int kKLoads = D == 128 ? kStepUnits : kStepUnits / 2;
  u32x4 kr[kKLoads];
  uint32_t ke[kKLoads];
  uint32_t vr[kStepUnits][4 * NE / 8];  // D = 128: a dword a row; 64: half of one
  uint32_t ve[kStepUnits];              // exponents of its four rows
  uint32_t mask[kStepUnits];
  const char *ku[kStepUnits], *vu[kStepUnits];  // (scalar)
  uint32_t eu[kStepUnits];
  auto locate = [&](int w) {  // units w, w + 1 of those held
#pragma unroll
    for (int i = 0; i < kStepUnits; ++i) {
      const uint32_t x = (uint32_t)__builtin_amdgcn_readlane(held_unit, w + i);
      mask[i] = (uint32_t)__builtin_amdgcn_readlane((int)held_mask, w + i);
      const uint32_t page = x >> unit_shift, in_page = x & ((1u << unit_shift) - 1u);
      const size_t at = (size_t)page * page_stride;
      ku[i] = k_head + at + in_page * kUnitBytes;
      vu[i] = v_head + at + in_page * kUnitBytes;
      eu[i] = exps_at - in_page * (kUnitBytes - kUnitExps);  // from a unit's codes to its exponents
    }
  };
  auto load_k = [&]() {
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < kStepUnits; ++i) {
        kr[i] = __builtin_nontemporal_load((global_u32x4)(uintptr_t)(ku[i] + 16u * (uint32_t)lane));
        ke[i] = *(global_u8)(uintptr_t)(ku[i] + eu[i] + (uint32_t)lane);
      }
    } else {
      const char* at = lane < 32 ? ku[0] : ku[1];
      const uint32_t l = (uint32_t)lane & 31u;
      kr[0] = __builtin_nontemporal_load((global_u32x4)(uintptr_t)(at + 16u * l));
      ke[0] = *(global_u8)(uintptr_t)(at + (lane < 32 ? eu[0] : eu[1]) + l);
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int i = 0; i < kStepUnits; ++i) {
      if constexpr (D == 128) {
        const u32x4 w = __builtin_nontemporal_load((global_u32x4)(uintptr_t)(vu[i] + 16u * (uint32_t)lane));
#pragma unroll
        for (int k = 0; k < 4; ++k) vr[i][k] = w[k];
      } else {
        const u32x2 w = __builtin_nontemporal_load((global_u32x2)(uintptr_t)(vu[i] + 8u * (uint32_t)lane));
        vr[i][0] = w[0];
        vr[i][1] = w[1];
      }
      ve[i] = *(global_u32)(uintptr_t)(vu[i] + eu[i] + 16u * (uint32_t)(qi * NE / kFp4Block) + 4u * (uint32_t)c4);
    }
  };

  i32x8 q_digits[kDigits];
  uint32_t q_exps[kDigits];
  auto load_queries = [&]() {
    const int block = D == 128 ? c4 : c4 & 1;
#pragma unroll
    for (int t = 0; t < kDigits; ++t) {
#pragma unroll
      for (int w = 0; w < 6; ++w) q_digits[t][w] = (int)s_u.q.digits[t][qi][block][w];
      q_digits[t][6] = q_digits[t][7] = 0;
      q_exps[t] = s_u.q.exps[t][qi][block];
    }
  };

  auto step = [&](bool more, int next) {
    // scores: sc[s][r] = column qi against row 4 c4 + r of unit s
    f32x4 sc[kStepUnits];
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
      i32x8 k = {0, 0, 0, 0, 0, 0, 0, 0};
      uint32_t e = ke[D == 128 ? s : 0];
#pragma unroll
      for (int w = 0; w < 4; ++w) k[w] = (int)kr[D == 128 ? s : 0][w];
      if constexpr (D == 64) {  // the other unit's lanes: zeros
        const bool here = (lane < 32) == (s == 0);
#pragma unroll
        for (int w = 0; w < 4; ++w) k[w] = here ? k[w] : 0;
        e = here ? e : 0u;
      }
      sc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = kDigits - 1; t >= 0; --t)
        sc[s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q_digits[t], sc[s], 4, 2, 0, (int)e, 0, (int)q_exps[t]);
    }
    uint32_t here[kStepUnits];
    bool plain = true;
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
      here[s] = mask[s];
      plain = plain && here[s] == 0xffffu;
    }
    if (more) {
      locate(next);
      load_k();
    }
    if (!plain) {
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) {
        const uint32_t rows = here[s] >> (4 * c4) & 15u;
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[s][r] = rows >> r & 1u ? sc[s][r] : -INFINITY;
        // an exponent that says NaN must not meet a weight of zero: codes of exponent 0 are finite
        const uint32_t bytes = (rows & 1u ? 0xffu : 0u) | (rows & 2u ? 0xff00u : 0u) | (rows & 4u ? 0xff0000u : 0u) | (rows & 8u ? 0xff000000u : 0u);
        ve[s] &= bytes;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[s][r]);
    }
    if (__builtin_amdgcn_ballot_w64(mx > ref) != 0) {
      mx = across_groups_max<16>(mx);
      const float ref_new = fmaxf(ref, mx), ref_safe = ref_new == -INFINITY ? 0.f : ref_new;
      const float alpha = __builtin_amdgcn_exp2f((ref - ref_safe) * post);
      ref = ref_new;
      lsum *= alpha;
#pragma unroll
      for (int e = 0; e < NE; ++e) O[e] *= alpha;
    }
    const float ref_safe = ref == -INFINITY ? 0.f : ref;
    uint32_t terms[kTerms][2 * kStepUnits];
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[s][r] = __builtin_amdgcn_exp2f((sc[s][r] - ref_safe) * post);
      lsum += (sc[s][0] + sc[s][1]) + (sc[s][2] + sc[s][3]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t tt[kTerms];
        BF16::template split<kTerms>(sc[s][2 * k], sc[s][2 * k + 1], tt);
#pragma unroll
        for (int i = 0; i < kTerms; ++i) terms[i][2 * s + k] = tt[i];
      }
    }
    // V: two channels of a row at a time, then two rows of a channel together
#pragma unroll
    for (int p = 0; p < NE / 2; ++p) {
      uint32_t two[kStepUnits][4];
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // (the conversion takes the exponent bits alone: what lies around them does not matter)
          const float scale = __builtin_bit_cast(float, r < 3 ? ve[s] << (23 - 8 * r) : ve[s] >> 1);
          if constexpr (D == 128) {
            two[s][r] = p == 0   ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vr[s][r], scale, 0))
                        : p == 1 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vr[s][r], scale, 1))
                        : p == 2 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vr[s][r], scale, 2))
                                 : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vr[s][r], scale, 3));
          } else {
            const uint32_t w = vr[s][r / 2];  // two rows of four channels
            const int byte = 2 * (r % 2) + p;
            two[s][r] = byte == 0   ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0))
                        : byte == 1 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1))
                        : byte == 2 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2))
                                    : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t sel = k ? 0x07060302u : 0x05040100u;
        const u32x4 v = {__builtin_amdgcn_perm(two[0][1], two[0][0], sel), __builtin_amdgcn_perm(two[0][3], two[0][2], sel),
                         __builtin_amdgcn_perm(two[1][1], two[1][0], sel), __builtin_amdgcn_perm(two[1][3], two[1][2], sel)};
#pragma unroll
        for (int i = kTerms - 1; i >= 0; --i) O[2 * p + k] = BF16::mfma(v, u32x4{terms[i][0], terms[i][1], terms[i][2], terms[i][3]}, O[2 * p + k]);
      }
    }
    if (more) load_v();
  };

  if (steps > 0) {
    find_units(0);
    locate(0);
    load_k();
    load_v();
  }
  __syncthreads();  // q's digits are laid out
  load_queries();
  for (int w = 0; w < steps * kStepUnits; w += kStepUnits) {
    const int next = w + kStepUnits;
    const bool more = next < steps * kStepUnits;
    if (more && next % kHeldUnits == 0) find_units(next);
    step(more, next % kHeldUnits);
  }
  lsum = across_groups_sum<16>(lsum);
  __syncthreads();  // q's digits are read by all: the states go where they were
  finish_pair<D, NE, false, false>(a, sl, h, ref, lsum, O, post, 1.f, s_ml, s_u.acc, s_ticket);
}

template <class Elt, int D, PagedKind kKind>
int run_fp4(const PagedArgs& base, const PagedPlan& p, const uint32_t* table, hipStream_t stream) {
  const dim3 grid((unsigned)base.heads, (unsigned)p.rows);
  if constexpr (kKind == kPagedSpans) {
    if (p.table) {
      PagedArgsTable a;
      static_cast<PagedArgs&>(a) = base;
      for (int32_t i = 0; i < p.rows; ++i) a.table[i] = table[i];
      hipLaunchKernelGGL((fp4_kernel<Elt, D, kKind, PagedArgsTable>), grid, dim3(kThreads), 0, stream, a);
      return launched();
    }
  }
  PagedArgsPlain a;
  static_cast<PagedArgs&>(a) = base;
  hipLaunchKernelGGL((fp4_kernel<Elt, D, kKind, PagedArgsPlain>), grid, dim3(kThreads), 0, stream, a);
  return launched();
}

template <PagedKind kKind>
int decode_fp4(const span_paged_desc_t* d, const void* q, const void* k, const void* v, const int32_t* block_table, const int32_t* ctx_lens,
               const int32_t* offsets, const int32_t* starts, const int32_t* ends, float scale, float* out) {
  PagedArgs a;
  PagedPlan p;
  uint32_t table[kMaxPlanSlices];
  const int rc = one_token_args(d, kKind, q, k, v, block_table, ctx_lens, offsets, starts, ends, nullptr, scale, nullptr, out, &a, &p, table);
  if (rc != SPAN_OK) return rc;
  hipStream_t stream = (hipStream_t)d->stream;
  const bool d128 = d->head_dim == 128;
  switch (d->dtype) {
    case SPAN_F32:
      return d128 ? run_fp4<F32, 128, kKind>(a, p, table, stream) : run_fp4<F32, 64, kKind>(a, p, table, stream);
    case SPAN_F16:
      return d128 ? run_fp4<F16, 128, kKind>(a, p, table, stream) : run_fp4<F16, 64, kKind>(a, p, table, stream);
    default:
      return d128 ? run_fp4<BF16, 128, kKind>(a, p, table, stream) : run_fp4<BF16, 64, kKind>(a, p, table, stream);
  }
}

}  // namespace
}  // namespace spanattn

extern "C" int paged_decode_attn_fp4(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                                     const int32_t* ctx_lens, float scale, float* out) {
  return spanattn::decode_fp4<spanattn::kPagedDense>(desc, q, k_pages, v_pages, block_table, ctx_lens, nullptr, nullptr, nullptr, scale, out);
}

extern "C" int paged_span_decode_attn_fp4(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                                          const int32_t* block_table, const int32_t* span_offsets, const int32_t* span_starts,
                                          const int32_t* span_ends, float scale, float* out) {
  return spanattn::decode_fp4<spanattn::kPagedSpans>(desc, q, k_pages, v_pages, block_table, nullptr, span_offsets, span_starts, span_ends, scale, out);
}
