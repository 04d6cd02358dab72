// One-token attention over a cache held in 4 bits, for up to 16 query heads per KV head.
//
// A workgroup of 4 wavefronts takes one slice of a (sequence, KV head) pair's positions and all query heads of the group, the columns of 16x16 matrix products; slices and the
// joining of states are those of the 16- and 32-bit caches (paged_attend.h).  What differs:
//   * Positions go in units of 16 aligned ones, which lie on one page: a unit's address and the mask of its rows are wave-uniform, found by the lanes 64 units at a
//     time, and every load is contiguous over the wave.  Where a window, a span or the cache begins or ends inside a unit, its other rows are masked; two intervals that meet in a unit are two units.
//   * K stays as it is: fp4 x fp6 products with both exponents applied by the matrix core.  q is laid out as kDigits digits to the base 16, each -16 .. 16 times a power of two that 32 channels share:
//     such a digit is an fp6 value (E2M3) exactly.  (The matrix core adds eight neighbouring products up with some 13 bits below the largest, measured; products of digits fit that, those of
//     floating values of different size do not.)  Five digits hold 21 bits below the largest channel of a block, six (fp32, or heads of 64) 25; of q below 2^-107 fewer.
//   * V becomes bf16, exactly, times its exponent: one instruction for two channels.  Weights meet it as three bf16 terms, all 24 bits.  (Two rounded terms leave 2^-18 of a weight, and outputs
//     2.4e-6 off in place of 1.4e-7, for 2 to 5 % of a call.)
//   * A step of 32 positions is bound by the instructions that a SIMD issues, not by the matrix core, and few heads leave columns free.  With up to 8 heads a head has two columns,
//     for even and odd channels: its weights go to every other of the product's inner places, zeros between them, and two channels of a row, as the conversion leaves them, need not be parted.  With up to 4
//     heads it has four, and two terms go through one product.
// What bounds it: memory where caches are even and large, else the start (launch, table entry, first rows: 5 us), the instructions of a SIMD's waves and the hand-over (3 us).  us, bytes over time: 64 x 8 pairs
// of 512 .. 4096 positions, four heads of 128 each, bf16 (166 MB, each byte fetched once) 37 .. 38, 4.4 TB/s, where slices of unlike length leave the longest to end alone (as many positions in level lengths, uncut: 30.5);
// 32 x 8 in a window of 4096 with 4 sinks (143 MB) 31 .. 32, 4.5 TB/s, 64 x 8 in one of 2048 28.7, 5.0 TB/s; 4 x 8 of 8000 .. 32768 (83 MB) 22.0 .. 22.5, 3.7 TB/s; 16 x 32 pairs of one head, ~500 positions in
// five spans, fp16 (42 MB, 49 fetched) 14.4 .. 15.4; four heads of 64 and 256 positions, fp32, 4.8; one sequence's 8 pairs in a window of 4096 10.9.
// Heads of 64 channels: two digits share a product with K, each half of the lanes has the rows (batch 27.7 -> 27.0, with fp32 queries 30.6 -> 29.2, the smallest call 4.88 -> 4.66; one digit and half a product of zeros
// before).  The rest of a step is as long as for 128.
#include "paged_attend.h"

namespace spanattn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef const SPAN_GLOBAL uint8_t* global_u8;
typedef const SPAN_GLOBAL uint32_t* global_u32;

constexpr int kUnitRows = kFp4Rows;
constexpr int kStepUnits = 2;                  // units that a wave takes together: 32 positions of one product with V
constexpr int kStepRows = kUnitRows * kStepUnits;
// The reference of the weights is moved on when a score's weight would pass 2^kSlack, not whenever the maximum moves: that is 57 instructions more in most of a wave's first steps.  (fp32 holds weights of 2^16 as exactly
// as those below 1, and a sum of 2^31 of them.)
constexpr float kSlack = 16.f;
// A page holds values up to 6 * 2^125, and up to 2^22 weights of 2^16 each would take a sum past fp32 whose mean is within.  From a wave's first block of V with an exponent of 65 or more on its
// weights stay 2^kLower below: 2^(16 - 40 + 22) of the largest values, and of those ahead 2^(16 + 22) below 2^68, are less than 2^126.  (What is below 2^-86 beside such a block loses bits.)
constexpr float kLower = 40.f;
constexpr int kHeldUnits = 64;                 // of a wave, found at a time: one per lane

template <class Elt, int D>
constexpr int kDigitsOf = Elt::kBytes == 4 || D == 64 ? 6 : 5;

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

// q in LDS: of each head and block of 32 channels the fp6 codes of every digit, and the digits' exponent bytes (of digit t byte t).
template <class Elt, int D>
struct DigitTables {
  uint32_t codes[kDigitsOf<Elt, D>][16][D / 32][6];
  uint8_t exps[16][D / 32][8];
};

// What a thread loads for its (block, digit) number i ...
template <class Elt, int D>
struct QueryBlock {
  static constexpr int kDigits = kDigitsOf<Elt, D>;
  u32x4 piece[2 * Elt::kBytes];
  __device__ __forceinline__ void load(const PagedArgs& a, size_t row0, int i) {
    const int block = i % (D / 32), j = i / (D / 32 * kDigits);
    const u32x4* from = (const u32x4*)((const char*)a.q + (row0 + (size_t)j) * (size_t)(D * Elt::kBytes) + (size_t)(block * 32 * Elt::kBytes));
#pragma unroll
    for (int p = 0; p < 2 * Elt::kBytes; ++p) piece[p] = from[p];
  }
  // ... and the digit's codes.
  __device__ __forceinline__ void lay(const PagedArgs& a, int i, DigitTables<Elt, D>& tab) {
    const int block = i % (D / 32), t = i / (D / 32) % kDigits, j = i / (D / 32 * kDigits);
    float x[32];
#pragma unroll
    for (int p = 0; p < 2 * Elt::kBytes; ++p) {
#pragma unroll
      for (int k = 0; k < 4; ++k) piece[p][k] = Elt::scale_query(piece[p][k], a.scale_log2e);
      Elt::unpack(piece[p], x + p * Elt::kPerVec);
    }
    float largest = 0.f;  // (NaN stays)
#pragma unroll
    for (int k = 0; k < 32; ++k) largest = __builtin_elementwise_maximum(largest, fabsf(x[k]));
    const uint32_t most = __builtin_bit_cast(uint32_t, largest) & 0x7fffffffu;
    // |x| < 2^(e - 126), e the largest's exponent bits; digit t counts 2^(e - 126 - 4 (t + 1)), as an fp6 value 8 times that each
    const int e = max((int)(most >> 23), 1);
    const int scale = e - 126 - 4 * (t + 1) + 3 + 127;
    tab.exps[j][block][t] = (uint8_t)(most >= 0x7f800000u ? 255 : max(scale, 0));  // (not finite: NaN)
    // What the digits ahead of this one leave, x less its nearest multiple of the last one's unit, is the digit times 2^-4 when rounded to a whole number of them: that is how
    // fp6 values up to 2 are spaced.  (Ties fall the same way for all threads.  The conversion takes its values from the two vectors in turn.)
    f32x16 half[2];
    const float ahead = t == 0 ? 0.f : -1.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      const float y = __builtin_amdgcn_ldexpf(x[k], 126 - e + 4 * t);
      half[k % 2][k / 2] = fmaf(rintf(y), ahead, y);
    }
    const u32x6 codes = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(half[0], half[1], 0.5f);
#pragma unroll
    for (int w = 0; w < 6; ++w) tab.codes[t][j][block][w] = scale < 0 ? 0u : codes[w];
  }
};

// sums += K (16 rows, fp4) x digit t of q (16 heads, fp6), both with their exponents.
__device__ __forceinline__ f32x4 digit_product(i32x8 k, int k_exp, i32x8 q, u32x2 q_exps, int t, f32x4 sums) {
  const int low = (int)q_exps[0], high = (int)q_exps[1];
  switch (t) {  // (which byte of the exponents is part of the instruction)
    case 0:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 0, low);
    case 1:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 1, low);
    case 2:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 2, low);
    case 3:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 3, low);
    case 4:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 0, high);
    default:
      return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q, sums, 4, 2, 0, k_exp, 1, high);
  }
}

// Waves whose registers hold the state, two steps' rows and the weights of one.
template <int D, int kShare>
constexpr int kFp4WavesPerSimd = D == 128 && kShare == 1 ? 3 : 4;

// kShare: columns that a query head has, 1, 2 or 4.
template <class Elt, int D, PagedKind kKind, int kShare, class Args>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kFp4WavesPerSimd<D, kShare>, kFp4WavesPerSimd<D, kShare>))) void fp4_kernel(const Args a) {
  constexpr bool kSpans = kKind == kPagedSpans;
  constexpr int kDigits = kDigitsOf<Elt, D>;
  constexpr int kProducts = D == 128 ? kDigits : kDigits / 2;  // of 128 inner places: one digit's channels, or two digits' 64
  constexpr int NE = D / 16;              // V channels of a lane
  constexpr int kHeads = 16 / kShare;     // heads that the columns hold
  constexpr int kSums = kShare == 1 ? NE : NE / 2;
  constexpr uint32_t kUnitBytes = 8u * D, kUnitExps = D / 2u;
  constexpr int kAccRow = D + 4;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qi = lane & 15, c4 = lane >> 4;
  const int h = blockIdx.x, kv_heads = a.heads, group = a.group;

  union Overlaid {
    DigitTables<Elt, D> q;
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
    sl = locate_slice(a, (int)blockIdx.y, lane, [&](int len) { return unit_count(seen_units(len, a.max_len, a.window, a.sinks)) * kUnitRows; });
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
  const float post = Elt::post_scale(a.scale_log2e);

  const int q_parts = group * (D / 32) * kDigits;  // (block, digit) pairs, a thread's at a time
  QueryBlock<Elt, D> q_block0;
  if (tid < q_parts) q_block0.load(a, bh * (size_t)group, tid);

  SeenUnits seen = {0, 0, 0, 0};
  int first_interval = 0, intervals = 0, all;  // units of the sequence
  struct Interval {
    int from, to, units;
  };
  Interval first_chunk = {0, 0, 0};  // of the sequence's first 64 intervals this lane's
  auto interval_of = [&](int i0) {   // of the 64 from i0 on
    Interval v = {0, 0, 0};
    if (i0 + lane < intervals) v.units = interval_units(a, a.starts[first_interval + i0 + lane], a.ends[first_interval + i0 + lane], v.from, v.to);
    return v;
  };
  if constexpr (kSpans) {
    const int lo = clampi(__builtin_amdgcn_readfirstlane(a.offsets[b]), 0, a.num_intervals);
    first_interval = lo;
    intervals = clampi(__builtin_amdgcn_readfirstlane(a.offsets[b + 1]), lo, a.num_intervals) - lo;
    all = 0;
    for (int i0 = 0; i0 < intervals; i0 += 64) {
      const Interval v = interval_of(i0);
      if (i0 == 0) first_chunk = v;
      all = min(all + __builtin_amdgcn_readlane(wave_inclusive_scan(v.units), 63), most_units(a, intervals));
    }
  } else {
    if (a.room == 0) sl.len = __builtin_amdgcn_readfirstlane(a.ctx_lens[b]);
    seen = seen_units(sl.len, a.max_len, a.window, a.sinks);
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

  // A wave's units, 64 at a time, one per lane: the page of the sequence that holds it, read from the table, its number on the page, and the mask of the rows that take part.
  struct Found {
    int page, at;
    uint32_t mask;
  };
  auto find_units = [&](int w0) {  // from the wave's unit w0 on
    const int w = w0 + lane, s = step0 + wave + w / kStepUnits * kWavesPerBlock;
    const int v = s * kStepUnits + w % kStepUnits;  // among the sequence's units
    const bool mine = w / kStepUnits < steps && v < all;
    int u = 0;
    Found f = {-1, 0, 0u};
    if constexpr (kSpans) {
      int before = 0;
      for (int i0 = 0; i0 < intervals; i0 += 64) {
        const Interval iv = i0 == 0 ? first_chunk : interval_of(i0);
        const int n = iv.units;
        const int incl = wave_inclusive_scan(n);
        // the first interval whose units end behind v
        int at = 0;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) {
          if (__shfl(incl, at + step - 1) + before <= v) at += step;
        }
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int ex = __shfl(incl - n, at), begin = __shfl(iv.from, at), end = __shfl(iv.to, at);
        if (mine && v >= before && v < before + total) {
          u = begin / kUnitRows + (v - before - ex);
          f.mask = unit_mask(u, begin, end);
        }
        before = min(before + total, most_units(a, intervals));
      }
    } else {
      const bool sink = v < seen.first;
      u = sink ? v : v - seen.first + seen.low / kUnitRows;
      if (mine) f.mask = unit_mask(u, sink ? 0 : seen.low, sink ? seen.sinks : seen.held);
    }
    if (mine && f.mask != 0) {
      f.page = table[u >> unit_shift];
      f.at = u & ((1 << unit_shift) - 1);
    }
    return f;
  };
  // Units of the pool (page * units of a page + unit in the page); none: the pool's first, which nobody attends.
  int held_unit = 0;
  uint32_t held_mask = 0;
  auto hold = [&](const Found& f) {
    const bool there = (uint32_t)f.page < (uint32_t)a.num_pages;
    held_mask = there ? f.mask : 0u;
    held_unit = there ? (f.page << unit_shift) + f.at : 0;
  };

  // A weight is exp2(score * post + shift): what the state is relative to is -shift as it is, rounded, and not the score that it came from.
  float shift = INFINITY, lsum = 0.f;
  bool large = false;  // a block of V that asks for kLower has been here
  // Unnormalised outputs.  kShare 1: O[e][r] of column qi's head, channel NE (4 c4 + r) + e.  Otherwise O[p][r], channel NE (4 c4 + r) + 2 p + odd; kShare 4: the term's part of it.
  f32x4 O[kSums];
#pragma unroll
  for (int e = 0; e < kSums; ++e) O[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int role = qi / kHeads;                    // of the column among its head's
  const bool odd = kShare > 1 && (role & 1);       // the channels that it sums
  const bool second = kShare == 4 && role >= 2;    // the second term's column: it brings the third too, in a product of its own
  const uint32_t taken = kShare == 4 && !second ? 0u : 0xffff0000u;  // of a weight ahead of the column's first term
  // Selector of a byte permutation: the upper half of a weight's rest, a bf16 value, to its place in the product's operand, zeros beside it; in columns without a third term, zeros alone.
  const uint32_t sel_place = odd ? 0x03020c0cu : 0x0c0c0302u, sel_last = kShare == 4 && !second ? 0x0c0c0c0cu : sel_place;

  // What a lane holds of a unit.  D = 128: K of row qi, channels 32 c4 on; D = 64: of two units together, K of row qi, unit c4 / 2, channels 32 (c4 % 2) on.  V of rows 4 c4 .. + 3, channels NE qi on.
  // A step's loads are under way while the step before it is worked on.
  constexpr int kKLoads = D == 128 ? kStepUnits : kStepUnits / 2;
  u32x4 kr[2][kKLoads];
  uint32_t ke[2][kKLoads];
  uint32_t vr[2][kStepUnits][4 * NE / 8];  // D = 128: a dword a row; 64: half of one
  uint32_t ve[2][kStepUnits];              // exponents of its four rows
  uint32_t mask[2][kStepUnits];
  auto fetch = [&](int w, auto place) {  // units w, w + 1 of those held
    constexpr int kTo = decltype(place)::value;
    const char SPAN_GLOBAL *ku[kStepUnits], *vu[kStepUnits];  // (scalar)
    uint32_t eu[kStepUnits];                                  // from a unit's codes to its exponents
    int ln = lane;
    asm volatile("" : "+v"(ln));  // (offsets are worked out here, next to the scalar addresses, and not kept)
    const uint32_t l = (uint32_t)ln;
    const uint32_t v_exp_off = 16u * ((l & 15u) * NE / kFp4Block) + 4u * (l >> 4);
#pragma unroll
    for (int i = 0; i < kStepUnits; ++i) {
      const uint32_t x = (uint32_t)__builtin_amdgcn_readlane(held_unit, w + i);
      mask[kTo][i] = (uint32_t)__builtin_amdgcn_readlane((int)held_mask, w + i);
      const uint32_t page = x >> unit_shift, in_page = x & ((1u << unit_shift) - 1u);
      const size_t at = (size_t)page * page_stride + in_page * kUnitBytes;
      ku[i] = (const char SPAN_GLOBAL*)(uintptr_t)(k_head + at);
      vu[i] = (const char SPAN_GLOBAL*)(uintptr_t)(v_head + at);
      eu[i] = exps_at - in_page * (kUnitBytes - kUnitExps);
    }
    if constexpr (D == 128) {
#pragma unroll
      for (int i = 0; i < kStepUnits; ++i) {
        kr[kTo][i] = __builtin_nontemporal_load((global_u32x4)(ku[i] + 16u * l));
        ke[kTo][i] = *(global_u8)(ku[i] + eu[i] + l);
      }
    } else {
      const char SPAN_GLOBAL* at = l < 32 ? ku[0] : ku[1];
      kr[kTo][0] = __builtin_nontemporal_load((global_u32x4)(at + 16u * (l & 31u)));
      ke[kTo][0] = *(global_u8)(at + (l < 32 ? eu[0] : eu[1]) + (l & 31u));
    }
#pragma unroll
    for (int i = 0; i < kStepUnits; ++i) {
      if constexpr (D == 128) {
        const u32x4 x = __builtin_nontemporal_load((global_u32x4)(vu[i] + 16u * l));
#pragma unroll
        for (int k = 0; k < 4; ++k) vr[kTo][i][k] = x[k];
      } else {
        const u32x2 x = __builtin_nontemporal_load((global_u32x2)(vu[i] + 8u * l));
        vr[kTo][i][0] = x[0];
        vr[kTo][i][1] = x[1];
      }
      ve[kTo][i] = *(global_u32)(vu[i] + eu[i] + v_exp_off);
    }
  };

  const int q_row = min(qi % kHeads, group - 1), q_block = D == 128 ? c4 : c4 & 1;  // (columns past the group are its last head's, never written)
  u32x2 q_exps = {0u, 0u};

  auto step = [&](auto place, bool more, int next) {
    constexpr int kAt = decltype(place)::value;
    auto& V = vr[kAt];
    auto& Ve = ve[kAt];
    if (more) fetch(next, std::integral_constant<int, 1 - kAt>());
    // scores: sc[s][r] = column qi against row 4 c4 + r of unit s.  A digit is read while the one before it is worked on, and not kept across the steps.
    f32x4 sc[kStepUnits];
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) sc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x8 digit[2];
    auto read_digit = [&](int t, i32x8& to) {  // of product t
      asm volatile("" ::: "memory");
#pragma unroll
      for (int w = 0; w < 6; ++w) to[w] = (int)s_u.q.codes[D == 128 ? t : 2 * t + c4 / 2][q_row][q_block][w];
      to[6] = to[7] = 0;
    };
    // (64: both halves of the lanes get a unit's rows, to meet a digit each)
    u32x4 rows[kStepUnits];
    uint32_t row_exps[kStepUnits];
    if constexpr (D == 128) {
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) rows[s] = kr[kAt][s], row_exps[s] = ke[kAt][s];
    } else {
      auto both = [](uint32_t x, uint32_t& low, uint32_t& high) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        low = r[0];
        high = r[1];
      };
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t low, high;
        both(kr[kAt][0][w], low, high);
        rows[0][w] = low;
        rows[1][w] = high;
      }
      both(ke[kAt][0], row_exps[0], row_exps[1]);
    }
    read_digit(kProducts - 1, digit[(kProducts - 1) & 1]);
#pragma unroll
    for (int t = kProducts - 1; t >= 0; --t) {
      if (t > 0) read_digit(t - 1, digit[(t - 1) & 1]);
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) {
        i32x8 k = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) k[w] = (int)rows[s][w];
        sc[s] = digit_product(k, (int)row_exps[s], digit[t & 1], q_exps, t, sc[s]);
      }
    }
    bool plain = true;
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) plain = plain && mask[kAt][s] == 0xffffu;
    if (!plain) {
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) {
        const uint32_t rows = mask[kAt][s] >> (4 * c4) & 15u;
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[s][r] = rows >> r & 1u ? sc[s][r] : -INFINITY;
        // an exponent that says NaN must not meet a weight of zero: codes of exponent 0 are finite
        const uint32_t bytes = (rows & 1u ? 0xffu : 0u) | (rows & 2u ? 0xff00u : 0u) | (rows & 4u ? 0xff0000u : 0u) | (rows & 8u ? 0xff000000u : 0u);
        Ve[s] &= bytes;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[s][r]);
    }
    const uint32_t upper_bits = (Ve[0] & Ve[0] << 1 | Ve[1] & Ve[1] << 1) & 0x80808080u;  // of an exponent byte from 192 on both
    large = large || __builtin_amdgcn_ballot_w64(upper_bits != 0u) != 0;
    const float lower = large ? kLower : 0.f;
    if (__builtin_amdgcn_ballot_w64(fmaf(mx, post, shift) > kSlack - lower) != 0) {
      mx = across_groups_max<16>(mx);
      const float to = fminf(shift, -(mx * post) - lower), to_safe = to == INFINITY ? 0.f : to;
      const float alpha = __builtin_amdgcn_exp2f(to_safe - shift);
      shift = to;
      lsum *= alpha;
#pragma unroll
      for (int e = 0; e < kSums; ++e) O[e] *= alpha;
    }
    const float shift_safe = shift == INFINITY ? 0.f : shift;
    // Weights as the products' operands, the smaller terms first: three times the upper half of what is left, eight bits each.  kShare 1: of all 32 rows, two in a dword; otherwise of a
    // unit's, one in a dword.
    constexpr int kPasses = kShare == 4 ? 2 : 3;
    u32x4 pairs[3], terms[kPasses][kStepUnits];
    auto less = [](float x, uint32_t mask) { return x - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & mask); };
    auto upper = [](float x, uint32_t sel) { return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), sel); };
#pragma unroll
    for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[s][r] = __builtin_amdgcn_exp2f(fmaf(sc[s][r], post, shift_safe));
      lsum += (sc[s][0] + sc[s][1]) + (sc[s][2] + sc[s][3]);
      if constexpr (kShare == 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float x = sc[s][2 * k], y = sc[s][2 * k + 1];
#pragma unroll
          for (int i = 2; i >= 0; --i) {
            pairs[i][2 * s + k] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, x), 0x07060302u);
            x = less(x, 0xffff0000u);
            y = less(y, 0xffff0000u);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = sc[s][r];
          if constexpr (kShare == 2) {
            terms[kPasses - 1][s][r] = upper(x, sel_place);
            x = less(x, 0xffff0000u);
          } else {
            x = less(x, taken);
          }
          terms[1][s][r] = upper(x, sel_place);
          terms[0][s][r] = upper(less(x, 0xffff0000u), sel_last);
        }
      }
    }
    // V: two channels of a row at a time
#pragma unroll
    for (int p = 0; p < NE / 2; ++p) {
      u32x4 two[kStepUnits];
#pragma unroll
      for (int s = 0; s < kStepUnits; ++s) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // (the conversion takes the exponent bits alone: what lies around them does not matter)
          const float scale = __builtin_bit_cast(float, r < 3 ? Ve[s] << (23 - 8 * r) : Ve[s] >> 1);
          const uint32_t w = D == 128 ? V[s][r] : V[s][r / 2];  // (64: two rows of four channels)
          const int byte = D == 128 ? p : 2 * (r % 2) + p;
          const bf16x2 v = byte == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)
                           : byte == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)
                           : byte == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)
                                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
          two[s][r] = __builtin_bit_cast(uint32_t, v);
        }
      }
      if constexpr (kShare == 1) {  // the two rows of a channel together
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t sel = k ? 0x07060302u : 0x05040100u;
          const u32x4 v = {__builtin_amdgcn_perm(two[0][1], two[0][0], sel), __builtin_amdgcn_perm(two[0][3], two[0][2], sel),
                           __builtin_amdgcn_perm(two[1][1], two[1][0], sel), __builtin_amdgcn_perm(two[1][3], two[1][2], sel)};
#pragma unroll
          for (int i = 0; i < 3; ++i) O[2 * p + k] = BF16::mfma(v, pairs[i], O[2 * p + k]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
#pragma unroll
          for (int s = 0; s < kStepUnits; ++s) O[p] = BF16::mfma(two[s], terms[i][s], O[p]);
        }
      }
    }
  };

  const Found first_units = find_units(0);
  if (tid < q_parts) q_block0.lay(a, tid, s_u.q);  // (while the table's entries are on their way)
  if (steps > 0) {
    hold(first_units);
    fetch(0, std::integral_constant<int, 0>());
  }
  for (int i = tid + kThreads; i < q_parts; i += kThreads) {
    QueryBlock<Elt, D> more;
    more.load(a, bh * (size_t)group, i);
    more.lay(a, i, s_u.q);
  }
  __syncthreads();
  q_exps = *reinterpret_cast<const u32x2*>(s_u.q.exps[q_row][q_block]);
  if constexpr (D == 64) q_exps[0] = __builtin_amdgcn_perm(q_exps[1], q_exps[0], c4 < 2 ? 0x0c040200u : 0x0c050301u);  // of the lane's digits
  const int units = steps * kStepUnits;
  auto next_of = [&](int w) {
    const int next = w + kStepUnits;
    if (next < units && next % kHeldUnits == 0) hold(find_units(next));
    return next;
  };
  for (int w = 0; w < units; w += 2 * kStepUnits) {
    int next = next_of(w);
    step(std::integral_constant<int, 0>(), next < units, next % kHeldUnits);
    if (next >= units) break;
    next = next_of(next);
    step(std::integral_constant<int, 1>(), next < units, next % kHeldUnits);
  }
  lsum = across_groups_sum<16>(lsum);
  __syncthreads();  // q's digits are read by all: the states go where they were
  if (c4 == 0 && qi < kHeads) s_ml[qi][wave] = f32x2{-shift, lsum};
  finish_pair<D, false, kShare>(a, sl, h, 1.f, 1.f, s_ml, s_u.acc, s_ticket, [&](float (&acc)[16][kAccRow]) {
    if constexpr (kShare == 4) {  // the terms' parts together
#pragma unroll
      for (int p = 0; p < kSums; ++p) {
#pragma unroll
        for (int r = 0; r < 4; ++r) O[p][r] += dpp_f<0x128>(O[p][r]);  // row_ror:8
      }
    }
    if (qi % kHeads >= group || second) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* row = &acc[qi % kHeads][NE * (4 * c4 + r)];
      if constexpr (kShare == 1) {
#pragma unroll
        for (int u = 0; u < NE / 4; ++u) *reinterpret_cast<f32x4*>(row + 4 * u) = f32x4{O[4 * u][r], O[4 * u + 1][r], O[4 * u + 2][r], O[4 * u + 3][r]};
      } else {
#pragma unroll
        for (int p = 0; p < kSums; ++p) row[2 * p + (odd ? 1 : 0)] = O[p][r];
      }
    }
  });
}

template <class Elt, int D, PagedKind kKind>
int run_fp4(const PagedArgs& base, const PagedPlan& p, const uint32_t* table, hipStream_t stream) {
  const dim3 grid((unsigned)base.heads, (unsigned)p.rows);
  auto start = [&](const auto& a) {
    using Args = std::decay_t<decltype(a)>;
    if (a.group > 8) hipLaunchKernelGGL((fp4_kernel<Elt, D, kKind, 1, Args>), grid, dim3(kThreads), 0, stream, a);
    else if (a.group > 4) hipLaunchKernelGGL((fp4_kernel<Elt, D, kKind, 2, Args>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((fp4_kernel<Elt, D, kKind, 4, Args>), grid, dim3(kThreads), 0, stream, a);
    return launched();
  };
  if constexpr (kKind == kPagedSpans) {
    if (p.table) {
      PagedArgsTable a;
      static_cast<PagedArgs&>(a) = base;
      for (int32_t i = 0; i < p.rows; ++i) a.table[i] = table[i];
      return start(a);
    }
  }
  PagedArgsPlain a;
  static_cast<PagedArgs&>(a) = base;
  return start(a);
}

template <PagedKind kKind>
int decode_fp4(const span_paged_desc_t* d, const void* q, const void* k, const void* v, const int32_t* block_table, const int32_t* ctx_lens,
               const int32_t* offsets, const int32_t* starts, const int32_t* ends, float scale, float* out) {
  PagedArgs a;
  PagedPlan p;
  uint32_t table[kMaxPlanSlices];
  const int rc = one_token_args(d, kKind, q, k, v, block_table, ctx_lens, offsets, starts, ends, nullptr, scale, nullptr, out, &a, &p, table, true);
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
