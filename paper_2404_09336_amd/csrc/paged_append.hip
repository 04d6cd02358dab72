// New rows into the pages with K (and q) turned by the angles of their positions, as they are or in 4 bits, and rows of 4-bit pages back as values.
//
// A pair of channels (x, x') becomes (x cos - x' sin, x sin + x' cos).  A wave takes a chunk of one token's rows, all of them of K, V and q in one launch; the rows are asked for first, and meanwhile
// the token's sequence, position, angles and page are found.  A lane's pieces of 16 bytes are at the same channels of every row, so that its angles are loaded once; the other channel of a pair
// comes from the lane that has it.
// What bounds it: memory where there are many rows.  Prompts of 16 sequences (32 + 2 * 8 rows of 128 channels a token, bf16, 517 MB read and written): 94.7 us, 5.5 TB/s, where a copy of 1 GiB
// reaches 5.06 on the same card.  64 rows of a step: 4.2 us, a launch's least with a chain of three trips (length, page and angles, stores).
// In 4 bits: 6 prompts, 5675 tokens of 2 * 32 rows of 128 and 32 of q, half of the channels turned in pairs, fp16 (211 MB read and written): 46 .. 47 us, 4.5 TB/s, where 41 are a copy's; 60 with all of
// them turned by halves; 21 .. 22 us to read them back (118 MB).  8133 such tokens without q (169 MB, a copy's 33): 44 turned in pairs or not at all, 57.5 by halves.  What is between: waves that all find their
// token, wait for angles and page and only then convert, 4 to 6 on a SIMD; those by halves have the other channels' values and both bounds of the error in registers too.  64 rows of a step 4.6 and 3.4 us.
#include "paged_device.h"

namespace spanattn {

namespace {

struct TokenArgs {
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* q_offsets;  // or null: row b is sequence b's
  const int32_t* seen;       // or null
  int32_t batch, table_pages, page_shift, num_pages, num_tokens, max_len;
};

struct TurnArgs : TokenArgs {
  const u32x4* k_new;
  const u32x4* v_new;
  const u32x4* q;            // or null
  void* k;                   // pools
  void* v;
  u32x4* q_out;
  int32_t* positions;        // or null
  const float* angles;       // [angle_rows, channels]: cosines, sines
  int32_t angle_rows, channels;  // channels 0: nothing is turned
  int32_t heads, kv_heads;
  int32_t chunks;                // waves that a token's rows take: those of K, then of V, then of q
};

struct ReadArgs : TokenArgs {
  const unsigned char* k;
  const unsigned char* v;
  u32x4* k_rows;
  u32x4* v_rows;
  int32_t kv_heads, chunks;
};

// A wave takes a chunk of so many pieces of 16 bytes per lane of one token's rows; a workgroup's waves the same chunk of neighbouring tokens, or neighbouring chunks.  Two a lane for a few tokens (more waves), twelve for
// many, the loads of a whole chunk under way together (with streamed stores and the other channel's values from their lane: the prompts above 121 -> 102 us); in 4 bits 2, 6 and 8 in place of four were
// no faster, sixteen waves a workgroup slower (53.7 -> 50.7 us for 8133 tokens of 2 * 32 rows of 128, fp16: with more than 64 registers a CU holds one of sixteen).
constexpr int kFewLoads = 2, kManyLoads = 12, kFp4Loads = 4;
constexpr int kWaves = 4, kFp4Waves = 8;
constexpr int32_t kManyTokens = 512;

// The sequence of a token's row, its slot and true position; b < 0: it belongs to none.
struct Token {
  int b, p, position;
};
__device__ __forceinline__ Token find_token(const TokenArgs& a, int t, int lane) {
  Token k = {t, 0, 0};
  int end = t + 1;
  if (a.q_offsets != nullptr) {
    k.b = sequence_of(a.q_offsets, a.batch, t, lane);
    if (k.b < 0 || a.q_offsets[k.b] > t) return Token{-1, 0, 0};
    end = a.q_offsets[k.b + 1];
  }
  k.b = __builtin_amdgcn_readfirstlane(k.b);
  const int len = a.ctx_lens[k.b];
  const uint32_t back = (uint32_t)t - (uint32_t)end;
  k.p = __builtin_amdgcn_readfirstlane((int)((uint32_t)len + back));
  k.position = __builtin_amdgcn_readfirstlane((int)((uint32_t)(a.seen != nullptr ? a.seen[k.b] : len) + back));
  return k;
}
// Row of the pool that a token has, -1: none.
__device__ __forceinline__ int token_row(const TokenArgs& a, const Token& k) {
  if ((uint32_t)k.p >= (uint32_t)a.max_len) return -1;
  return __builtin_amdgcn_readfirstlane(pool_row(a.block_table + (size_t)k.b * a.table_pages, k.p, a.page_shift, a.num_pages));
}

template <class Elt>
__device__ __forceinline__ u32x4 pack_values(const float* f) {
  u32x4 r;
  if constexpr (Elt::kBytes == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = Elt::pack2(f[2 * i], f[2 * i + 1]);
  }
  return r;
}

// The angles of a lane's channels, the same for every row that it takes: cosines and sines, the latter with the sign that the other channel of a pair has.
template <class Elt, bool kPaired>
struct Angles {
  static constexpr int kPer = Elt::kPerVec, kOwn = kPaired ? kPer / 2 : kPer;
  float cosine[kOwn], sine[kOwn];
  int partner;  // halves: lanes from a lane's piece to that of the other channels
  bool turned;

  __device__ __forceinline__ void load(const TurnArgs& a, int position, int piece) {
    const int d = piece * kPer, half = a.channels / 2;
    turned = d < a.channels;
    partner = 0;
    if (!turned) return;
    const bool second = !kPaired && d >= half;
    const int first = kPaired ? d / 2 : d - (second ? half : 0);
    partner = (second ? -half : half) / kPer;
    const bool known = (uint32_t)position < (uint32_t)a.angle_rows;
    const float* row = a.angles + (size_t)(known ? position : 0) * (size_t)a.channels + first;
    // (the table's rows are whole lines of 64 bytes, halves of 32; one number at a time took 102 us in place of 95 for the prompts above, in 4 bits 80 in place of 60 for 8133 tokens turned by halves)
    constexpr int kWide = kOwn < 4 ? kOwn : 4;
    typedef float Wide __attribute__((ext_vector_type(kWide)));
    Wide c[kOwn / kWide], s[kOwn / kWide];
#pragma unroll
    for (int i = 0; i < kOwn / kWide; ++i) c[i] = *(const Wide*)(row + kWide * i), s[i] = *(const Wide*)(row + half + kWide * i);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      const float sin = s[i / kWide][i % kWide];
      cosine[i] = known ? c[i / kWide][i % kWide] : NAN;
      sine[i] = known ? (second || kPaired ? sin : -sin) : NAN;
    }
  }
};

// y = x cos + x' sin (the sine's sign is x's own); paired: both of a pair are here.
template <class Elt, bool kPaired>
__device__ __forceinline__ void turn(const Angles<Elt, kPaired>& g, float* x, const float* other) {
#pragma unroll
  for (int i = 0; i < Elt::kPerVec; ++i) {
    if constexpr (kPaired) {
      if (i & 1) continue;
      const float one = x[i], two = x[i + 1];
      x[i] = fmaf(one, g.cosine[i / 2], -(two * g.sine[i / 2]));
      x[i + 1] = fmaf(one, g.sine[i / 2], two * g.cosine[i / 2]);
    } else {
      x[i] = fmaf(x[i], g.cosine[i], other[i] * g.sine[i]);
    }
  }
}

// x to fp32, inexact values to the neighbour with an odd last bit: rounded again to fewer bits, with ties to even, it becomes what x would.  kTiny: also below 2^-126, where
// fp32 has fewer bits than the 24 that are kept otherwise.
template <bool kTiny>
__device__ __forceinline__ float to_odd(double x) {
  if constexpr (kTiny) {
    const float f = (float)x;
    const double back = (double)f;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (fabs(back) > fabs(x)) u -= 1u;
    if (back != x) u |= 1u;
    return __builtin_bit_cast(float, u);
  }
  u32x2 u = __builtin_bit_cast(u32x2, x);
  u[0] = (u[0] & 0xe0000000u) | min(u[0] & 0x1fffffffu, 1u) << 29;
  return (float)__builtin_bit_cast(double, u);
}
// The same as turn, to the odd neighbour of the exact value: products of two fp32 are exact in 64 bits, their sum is rounded once.
template <class Elt, bool kPaired, bool kTiny>
__device__ __forceinline__ void turn_exactly(const Angles<Elt, kPaired>& g, float* x, const float* other) {
#pragma unroll
  for (int i = 0; i < Elt::kPerVec; ++i) {
    if constexpr (kPaired) {
      if (i & 1) continue;
      const double one = x[i], two = x[i + 1], c = g.cosine[i / 2], s = g.sine[i / 2];
      x[i] = to_odd<kTiny>(fma(one, c, -(two * s)));
      x[i + 1] = to_odd<kTiny>(fma(one, s, two * c));
    } else {
      x[i] = to_odd<kTiny>(fma((double)x[i], (double)g.cosine[i], (double)other[i] * (double)g.sine[i]));
    }
  }
}

// The largest of the lanes that hold a block of 32 channels together, kPer each; values not below zero as bits (NaN above infinity above numbers).
template <int kPer>
__device__ __forceinline__ uint32_t block_most(uint32_t most) {
  most = max(most, (uint32_t)dpp_i<0xB1>((int)most));            // quad_perm [1,0,3,2]
  most = max(most, (uint32_t)dpp_i<0x4E>((int)most));            // quad_perm [2,3,0,1]
  if (kPer == 4) most = max(most, (uint32_t)dpp_i<0x141>((int)most));  // row_half_mirror
  return most;
}
// Exponent byte of a block by its largest magnitude.
__device__ __forceinline__ uint32_t exponent_of(uint32_t most) {
  constexpr uint32_t kSeven = 0x00600000u;                       // mantissa of 7 = 1.75 * 2^2
  constexpr uint32_t kMost = ((uint32_t)(kFp4MostExponent + 2 + 127) << 23) | kSeven;
  if (most > kMost) return 255u;
  const int e = (int)(most >> 23) - 2 + ((most & 0x7fffffu) > kSeven ? 1 : 0);  // e + 127
  return (uint32_t)max(e, kFp4LeastExponent + 127);
}
template <int kPer>
__device__ __forceinline__ float largest_of(const float* x) {  // (NaN stays)
  float largest = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) largest = __builtin_elementwise_maximum(largest, fabsf(x[i]));
  return fabsf(largest);
}
template <int kPer>
__device__ __forceinline__ uint32_t block_exponent(const float* x) {
  return exponent_of(block_most<kPer>(__builtin_bit_cast(uint32_t, largest_of<kPer>(x))));
}

// Codes of 4 kPairs / 2 ... values by a block's exponent, the first in the lowest four bits.  (The instruction takes the scale's exponent alone, rounds to the nearest, ties to the even code, and
// cuts off at 6.)
template <int kPer>
__device__ __forceinline__ uint32_t to_codes(const float* x, uint32_t exponent) {
  const float scale = __builtin_bit_cast(float, exponent << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  if constexpr (kPer == 8) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  }
  return w;
}

// Where four channels of a row lie on a page of 4-bit values, and the exponent of their block.
template <int D, bool kV>
__device__ __forceinline__ uint32_t code_at(uint32_t row, uint32_t c) {
  constexpr uint32_t w = D / 16;
  const uint32_t group = row / kFp4Rows, r = row % kFp4Rows;
  if constexpr (kV) return group * (8u * D) + r / 4u * (2u * D) + c / w * (2u * w) + r % 4u * (w / 2u) + c % w / 2u;
  return group * (8u * D) + c / 32u * 256u + r * 16u + c % 32u / 2u;
}
template <int D>
__device__ __forceinline__ uint32_t exponent_at(uint32_t page_rows, uint32_t row, uint32_t c) {
  return page_rows * (D / 2u) + row / kFp4Rows * (D / 2u) + c / 32u * 16u + row % kFp4Rows;
}

// Bound by memory where there are many rows, by the chain of trips (offsets, length, angles and page) where there are few.
template <class Elt, int D, bool kFp4, bool kPaired, int kLoads>
__global__ __launch_bounds__(64 * (kFp4 ? kFp4Waves : kWaves)) void turn_kernel(const TurnArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;  // pieces of a row
  constexpr int kChunk = 64 * kLoads;
  // Many tokens' 4-bit rows go out by way of LDS, so that neighbouring lanes store what neighbouring tokens have in a line: 16 bytes of K, 4 of V where a row by itself is stored by 4 and 1 (those
  // tokens 59.6 -> 53.7 us).
  constexpr bool kStaged = kFp4 && kLoads == kFp4Loads;
  constexpr int kTokenCodes = kChunk * kPer / 2, kTokenExps = kChunk * kPer / kFp4Block;  // bytes of a token's chunk
  __shared__ __attribute__((aligned(16))) unsigned char s_codes[kStaged ? kFp4Waves : 1][kStaged ? kTokenCodes + 16 : 16];
  __shared__ unsigned char s_exps[kStaged ? kFp4Waves : 1][kStaged ? kTokenExps + 4 : 4];
  __shared__ int s_rows[kFp4Waves];  // of the pool that the tokens have, or -1
  const int lane = threadIdx.x & 63;
  const uint32_t chunks = (uint32_t)a.chunks, waves = blockDim.x >> 6, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint32_t unit = blockIdx.x * waves + wave;
  const int t = kFp4 ? (int)(blockIdx.x / chunks * waves + wave) : (int)(unit / chunks), c = kFp4 ? (int)(blockIdx.x % chunks) : (int)(unit % chunks);
  if constexpr (kStaged) {
    if (lane == 0) s_rows[wave] = -1;  // (until it is known: what returns ahead of the barrier's wait has no row)
  } else {
    if (t >= a.num_tokens) return;
  }
  const int rows = 2 * a.kv_heads + (a.q != nullptr ? a.heads : 0), pieces = rows * kRow;
  const int first = c * kChunk + lane, piece = lane % kRow;
  // Row number `row` of a token: of K, of V or of q, where it begins.
  auto source = [&](int row) {
    const bool is_q = row >= 2 * a.kv_heads, is_v = row >= a.kv_heads;
    const u32x4* of = is_q ? a.q : is_v ? a.v_new : a.k_new;
    const int heads = is_q ? a.heads : a.kv_heads, h = row - (is_q ? 2 * a.kv_heads : is_v ? a.kv_heads : 0);
    return of + ((size_t)t * (size_t)heads + (size_t)h) * (size_t)kRow;
  };
  auto whole_or_part = [&](auto whole) {  // (a whole chunk's loads are not parted by branches)
    constexpr bool kWhole = decltype(whole)::value;
    u32x4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (!kWhole && c * kChunk + 64 * i >= pieces) break;
      const int at = kWhole ? first + 64 * i : min(first + 64 * i, pieces - 1);
      x[i] = __builtin_nontemporal_load(source(at / kRow) + piece);
    }
    const Token tok = find_token(a, t, lane);
    if (tok.b < 0) return;
    Angles<Elt, kPaired> g;
    g.turned = false;
    g.partner = 0;
    const bool only_v = c * kChunk >= a.kv_heads * kRow && (c + 1) * kChunk <= 2 * a.kv_heads * kRow;
    if (a.channels > 0 && !only_v) g.load(a, tok.position, piece);
    float most_angle = 0.f;  // ... times 2^-21
    if (kFp4 && g.turned) most_angle = 0x1p-21f * __builtin_elementwise_maximum(largest_of<Angles<Elt, kPaired>::kOwn>(g.cosine), largest_of<Angles<Elt, kPaired>::kOwn>(g.sine));
    if (c == 0 && a.positions != nullptr && (uint32_t)tok.p < (uint32_t)a.max_len) {
      for (int h = lane; h < a.kv_heads; h += 64) a.positions[((size_t)tok.b * a.kv_heads + h) * (size_t)a.max_len + tok.p] = tok.position;
    }
    const int at_row = c * kChunk < 2 * a.kv_heads * kRow ? token_row(a, tok) : -1;  // of the pool (a chunk of q needs none)
    const size_t page = (size_t)(max(at_row, 0) >> a.page_shift);
    const uint32_t page_rows = 1u << a.page_shift, in_page = (uint32_t)max(at_row, 0) & (page_rows - 1u);
    if (kStaged && lane == 0) s_rows[wave] = at_row;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (!kWhole && c * kChunk + 64 * i >= pieces) break;
      const int at = first + 64 * i, row = at / kRow;
      const bool is_q = row >= 2 * a.kv_heads, is_v = !is_q && row >= a.kv_heads;
      const int h = row - (is_q ? 2 * a.kv_heads : is_v ? a.kv_heads : 0);
      const bool turned = g.turned && !is_v;
      float f[kPer], o[kPer];
      Elt::unpack(x[i], f);
      if (!kPaired && a.channels > 0 && !only_v) {  // (of every lane: the other channels' values come from theirs)
        u32x4 other;
#pragma unroll
        for (int k = 0; k < 4; ++k) other[k] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane + g.partner), (int)x[i][k]);
        Elt::unpack(other, o);
      }
      if (kFp4 && !is_q) {
        uint32_t exponent, w;
        bool sure = false;
        if (a.channels > 0 && !only_v) {
          // In fp32 the turned values are less than `off` away: two products and a sum of 2^-24 each, at most 3 of them, and 2 for the sums with `off`, times the largest x times the largest angle; 8 are
          // taken.  Where all that may be has one exponent and one code, those are the exact values' too.
          float y[kPer], low[kPer], high[kPer], off = 0.f;
#pragma unroll
          for (int k = 0; k < kPer; ++k) y[k] = f[k];
          bool within = true;
          if (turned) {
            off = largest_of<kPer>(f);
            if constexpr (!kPaired) off = __builtin_elementwise_maximum(off, largest_of<kPer>(o));
            off *= most_angle;
            within = off >= 0x1p-100f && off <= 0x1p+100f;  // (of others, fp32's least numbers and overflow among them, nothing is said)
            turn<Elt, kPaired>(g, y, o);
          }
          const float most = largest_of<kPer>(y);
          const float least_most = within ? __builtin_elementwise_maximum(most - off, 0.f) : 0.f, most_most = within ? most + off : INFINITY;
          exponent = exponent_of(block_most<kPer>(__builtin_bit_cast(uint32_t, most_most)));  // (a block's lanes are all here)
          sure = exponent == exponent_of(block_most<kPer>(__builtin_bit_cast(uint32_t, least_most)));
#pragma unroll
          for (int k = 0; k < kPer; ++k) low[k] = y[k] - off, high[k] = y[k] + off;
          w = to_codes<kPer>(high, exponent);
          sure = sure && w == to_codes<kPer>(low, exponent);
        }
        if (__builtin_amdgcn_ballot_w64(!sure) != 0) {
#pragma unroll
          for (int k = 0; k < Angles<Elt, kPaired>::kOwn; ++k) asm volatile("" : "+v"(g.cosine[k]), "+v"(g.sine[k]));  // (not kept as 64-bit numbers beside)
          if (turned) turn_exactly<Elt, kPaired, false>(g, f, o);
          exponent = block_exponent<kPer>(f);
          if (turned && exponent <= kFp4LeastExponent + 128) {  // (from the next exponent on the least border, a quarter, is one of fp32's numbers of 24 bits)
            Elt::unpack(x[i], f);
            turn_exactly<Elt, kPaired, true>(g, f, o);
          }
          w = to_codes<kPer>(f, exponent);
        }
        if constexpr (kStaged) {
          const int here = 64 * i + lane;
          if constexpr (kPer == 8) *(uint32_t*)&s_codes[wave][4 * here] = w;
          else *(uint16_t*)&s_codes[wave][2 * here] = (uint16_t)w;
          if (here * kPer % kFp4Block == 0) s_exps[wave][here * kPer / kFp4Block] = (unsigned char)exponent;
        } else if (at_row >= 0 && (kWhole || at < pieces)) {
          const uint32_t ch = (uint32_t)piece * kPer;
          unsigned char* to = (unsigned char*)(is_v ? a.v : a.k) + (page * (size_t)a.kv_heads + (size_t)h) * ((size_t)page_rows * (D / 2 + D / kFp4Block));
          const uint32_t code = is_v ? code_at<D, true>(in_page, ch) : code_at<D, false>(in_page, ch);
          if constexpr (kPer == 8 && D == 128) {
            *(uint32_t*)(to + code) = w;
          } else if constexpr (kPer == 8) {
            *(uint16_t*)(to + code) = (uint16_t)w;
            *(uint16_t*)(to + (is_v ? code_at<D, true>(in_page, ch + 4u) : code + 2u)) = (uint16_t)(w >> 16);
          } else {
            *(uint16_t*)(to + code) = (uint16_t)w;
          }
          if (ch % kFp4Block == 0) to[exponent_at<D>(page_rows, in_page, ch)] = (unsigned char)exponent;
        }
        continue;
      }
      if (turned) {
        turn<Elt, kPaired>(g, f, o);
        x[i] = pack_values<Elt>(f);
      }
      if (!kWhole && at >= pieces) continue;
      if (is_q) {
        __builtin_nontemporal_store(x[i], a.q_out + ((size_t)t * (size_t)a.heads + (size_t)h) * (size_t)kRow + (size_t)piece);
      } else if (!kFp4 && at_row >= 0) {
        const size_t to = (((page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) + in_page) * (size_t)kRow + (size_t)piece;
        __builtin_nontemporal_store(x[i], (u32x4*)(is_v ? a.v : a.k) + to);
      }
    }
  };
  if (!kStaged || t < a.num_tokens) {
    if ((c + 1) * kChunk <= pieces) whole_or_part(std::true_type());
    else whole_or_part(std::false_type());
  }
  if constexpr (kStaged) {
    constexpr int kRows = kChunk / kRow, kBlocks = D / kFp4Block, w = D / 16;  // rows of the chunk; w: channels that V has of a row in one place
    const int row0 = c * kRows, end = min(kRows, 2 * a.kv_heads - row0);       // (rows of q from there on)
    if (end <= 0) return;
    __syncthreads();
    const uint32_t page_rows = 1u << a.page_shift;
    auto head_of = [&](int at_row, int row) {  // where a row's (page, head) begins
      const bool is_v = row >= a.kv_heads;
      return (unsigned char*)(is_v ? a.v : a.k) + ((size_t)(at_row >> a.page_shift) * (size_t)a.kv_heads + (size_t)(is_v ? row - a.kv_heads : row)) * ((size_t)page_rows * (D / 2 + D / kFp4Block));
    };
    for (int i = (int)threadIdx.x; i < end * kBlocks * kFp4Waves; i += 64 * kFp4Waves) {
      const int token = i % kFp4Waves, block = i / kFp4Waves % kBlocks, r = i / (kFp4Waves * kBlocks), row = row0 + r, at_row = s_rows[token];
      if (at_row < 0) continue;
      unsigned char* to = head_of(at_row, row);
      const uint32_t in_page = (uint32_t)at_row & (page_rows - 1u);
      to[exponent_at<D>(page_rows, in_page, (uint32_t)block * kFp4Block)] = s_exps[token][r * kBlocks + block];
      if (row < a.kv_heads) *(u32x4*)(to + code_at<D, false>(in_page, (uint32_t)block * kFp4Block)) = *(const u32x4*)&s_codes[token][r * (D / 2) + block * (kFp4Block / 2)];
    }
    const int first_v = max(a.kv_heads - row0, 0);
    for (int i = (int)threadIdx.x; i < (end - first_v) * 16 * kFp4Waves; i += 64 * kFp4Waves) {
      const int token = i % 4 + i / 64 % (kFp4Waves / 4) * 4, part = i / 4 % 16, r = first_v + i / (16 * kFp4Waves), at_row = s_rows[token];
      if (at_row < 0) continue;
      const uint32_t in_page = (uint32_t)at_row & (page_rows - 1u);
      unsigned char* to = head_of(at_row, row0 + r) + code_at<D, true>(in_page, (uint32_t)(part * w));
      const unsigned char* from = &s_codes[token][r * (D / 2) + part * (w / 2)];
      if constexpr (w == 8) *(uint32_t*)to = *(const uint32_t*)from;
      else *(uint16_t*)to = *(const uint16_t*)from;
    }
  }
}

template <class Elt, int D>
__global__ __launch_bounds__(64 * kFp4Waves) void read_kernel(const ReadArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;
  const int lane = threadIdx.x & 63;
  const uint32_t chunks = (uint32_t)a.chunks, waves = blockDim.x >> 6;
  const int c = (int)(blockIdx.x % chunks);
  const int t = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / chunks * waves + (threadIdx.x >> 6)));
  if (t >= a.num_tokens) return;
  const Token tok = find_token(a, t, lane);
  if (tok.b < 0) return;
  const int at_row = token_row(a, tok);
  if (at_row < 0) return;
  const size_t page = (size_t)(at_row >> a.page_shift);
  const uint32_t page_rows = 1u << a.page_shift, in_page = (uint32_t)at_row & (page_rows - 1u);
  const int pieces = 2 * a.kv_heads * kRow, piece = lane % kRow;
  const uint32_t ch = (uint32_t)piece * kPer;
  uint32_t w[kFp4Loads], exponent[kFp4Loads];
#pragma unroll
  for (int i = 0; i < kFp4Loads; ++i) {
    const int row = min(c * (64 * kFp4Loads) + lane + 64 * i, pieces - 1) / kRow;
    const bool is_v = row >= a.kv_heads;
    const unsigned char* of =
        (is_v ? a.v : a.k) + (page * (size_t)a.kv_heads + (size_t)(is_v ? row - a.kv_heads : row)) * ((size_t)page_rows * (D / 2 + D / kFp4Block));
    const uint32_t code = is_v ? code_at<D, true>(in_page, ch) : code_at<D, false>(in_page, ch);
    exponent[i] = of[exponent_at<D>(page_rows, in_page, ch)];
    if constexpr (kPer == 8 && D == 128) w[i] = *(const uint32_t*)(of + code);
    else if constexpr (kPer == 8) w[i] = *(const uint16_t*)(of + code) | (uint32_t) * (const uint16_t*)(of + (is_v ? code_at<D, true>(in_page, ch + 4u) : code + 2u)) << 16;
    else w[i] = *(const uint16_t*)(of + code);
  }
#pragma unroll
  for (int i = 0; i < kFp4Loads; ++i) {
    const int at = c * (64 * kFp4Loads) + lane + 64 * i, row = at / kRow;
    const bool is_v = row >= a.kv_heads;
    const float scale = __builtin_bit_cast(float, exponent[i] << 23);
    float f[8];
    f32x2 two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 0);
    f[0] = two[0], f[1] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 1);
    f[2] = two[0], f[3] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 2);
    f[4] = two[0], f[5] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i], scale, 3);
    f[6] = two[0], f[7] = two[1];
    if (at < pieces)
      (is_v ? a.v_rows : a.k_rows)[((size_t)t * (size_t)a.kv_heads + (size_t)(is_v ? row - a.kv_heads : row)) * (size_t)kRow + (size_t)piece] = pack_values<Elt>(f);
  }
}

TokenArgs token_args(const span_paged_desc_t* d, const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* seen) {
  TokenArgs a = {};
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.q_offsets = q_offsets;
  a.seen = seen;
  a.batch = d->batch;
  a.table_pages = d->table_pages;
  a.page_shift = page_shift(d);
  a.num_pages = d->num_pages;
  a.num_tokens = d->num_tokens;
  a.max_len = capacity(d);
  return a;
}

// Chunks of so many loads that `rows` rows of a token take.
int64_t chunks_of(const span_paged_desc_t* d, int64_t rows, int loads) {
  const int64_t pieces = rows * (d->head_dim * (d->dtype == SPAN_F32 ? 4 : 2) / 16);
  return (pieces + 64 * loads - 1) / (64 * loads);
}

struct TokenGrid {
  dim3 grid, block;
};
// Grid of so many waves a token; false: 2^32 lanes or more.
bool grid_of(const span_paged_desc_t* d, int64_t chunks, int waves, TokenGrid* g) {
  const int64_t groups = ((int64_t)d->num_tokens + waves - 1) / waves * chunks;
  if (groups * waves > 0x3ffffff) return false;
  g->grid = dim3((unsigned)groups);
  g->block = dim3((unsigned)(64 * waves));
  return true;
}

template <class Elt, int D, bool kFp4>
void start_turn(const TurnArgs& a, bool paired, bool many, const TokenGrid& g, hipStream_t stream) {
  constexpr int kMany = kFp4 ? kFp4Loads : kManyLoads;
  auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, g.grid, g.block, 0, stream, a); };
  if (many) paired ? start(turn_kernel<Elt, D, kFp4, true, kMany>) : start(turn_kernel<Elt, D, kFp4, false, kMany>);
  else paired ? start(turn_kernel<Elt, D, kFp4, true, kFewLoads>) : start(turn_kernel<Elt, D, kFp4, false, kFewLoads>);
}

template <bool kFp4>
int append_turned(const span_paged_desc_t* d, const paged_rotation_t* rotation, const void* k_new, const void* v_new, void* k, void* v,
                  const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, int32_t* positions, const int32_t* seen, const void* q,
                  void* q_out) {
  int rc = check_paged(d);
  if (rc != SPAN_OK) return rc;
  if (!kFp4 && !rotation) return SPAN_ERR_NULL;
  rc = check_rotation(d, rotation);
  if (rc != SPAN_OK) return rc;
  if (!q != !q_out) return SPAN_ERR_NULL;
  if (!q_offsets && d->num_tokens != 0 && d->num_tokens != d->batch) return SPAN_ERR_SHAPE;
  if (d->num_tokens == 0) return SPAN_OK;
  if (!k_new || !v_new || !k || !v || !block_table || !ctx_lens) return SPAN_ERR_NULL;
  TurnArgs a = {};
  static_cast<TokenArgs&>(a) = token_args(d, block_table, ctx_lens, q_offsets, seen);
  a.k_new = (const u32x4*)k_new;
  a.v_new = (const u32x4*)v_new;
  a.q = (const u32x4*)q;
  a.k = k;
  a.v = v;
  a.q_out = (u32x4*)q_out;
  a.positions = positions;
  if (rotation) {
    a.angles = rotation->table;
    a.angle_rows = rotation->positions;
    a.channels = rotation->channels;
  }
  a.heads = d->heads;
  a.kv_heads = d->kv_heads;
  const bool many = d->num_tokens >= kManyTokens;
  const int64_t chunks = chunks_of(d, 2 * (int64_t)d->kv_heads + (q ? d->heads : 0), !many ? kFewLoads : kFp4 ? kFp4Loads : kManyLoads);
  TokenGrid grid;
  if (!grid_of(d, chunks, kFp4 && many ? kFp4Waves : kWaves, &grid)) return SPAN_ERR_SHAPE;
  a.chunks = (int32_t)chunks;
  const bool paired = !rotation || rotation->paired, d128 = d->head_dim == 128;
  hipStream_t stream = (hipStream_t)d->stream;
  switch (d->dtype) {
    case SPAN_F32:
      d128 ? start_turn<F32, 128, kFp4>(a, paired, many, grid, stream) : start_turn<F32, 64, kFp4>(a, paired, many, grid, stream);
      break;
    case SPAN_F16:
      d128 ? start_turn<F16, 128, kFp4>(a, paired, many, grid, stream) : start_turn<F16, 64, kFp4>(a, paired, many, grid, stream);
      break;
    default:
      d128 ? start_turn<BF16, 128, kFp4>(a, paired, many, grid, stream) : start_turn<BF16, 64, kFp4>(a, paired, many, grid, stream);
  }
  return launched();
}

}  // namespace
}  // namespace spanattn

extern "C" int paged_append_rotary(const span_paged_desc_t* desc, const paged_rotation_t* rotation, const void* k_new, const void* v_new, void* k_pages,
                                   void* v_pages, const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, int32_t* positions,
                                   const int32_t* seen, const void* q, void* q_out) {
  return spanattn::append_turned<false>(desc, rotation, k_new, v_new, k_pages, v_pages, block_table, ctx_lens, q_offsets, positions, seen, q, q_out);
}

extern "C" int paged_append_fp4(const span_paged_desc_t* desc, const paged_rotation_t* rotation, const void* k_new, const void* v_new, void* k_pages,
                                void* v_pages, const int32_t* block_table, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* seen,
                                const void* q, void* q_out) {
  return spanattn::append_turned<true>(desc, rotation, k_new, v_new, k_pages, v_pages, block_table, ctx_lens, q_offsets, nullptr, seen, q, q_out);
}

extern "C" int paged_read_fp4(const span_paged_desc_t* desc, const void* k_pages, const void* v_pages, const int32_t* block_table,
                              const int32_t* ctx_lens, const int32_t* q_offsets, void* k_rows, void* v_rows) {
  using namespace spanattn;
  const int rc = check_paged(desc);
  if (rc != SPAN_OK) return rc;
  if (!q_offsets && desc->num_tokens != 0 && desc->num_tokens != desc->batch) return SPAN_ERR_SHAPE;
  if (desc->num_tokens == 0) return SPAN_OK;
  if (!k_pages || !v_pages || !block_table || !ctx_lens || !k_rows || !v_rows) return SPAN_ERR_NULL;
  ReadArgs a = {};
  static_cast<TokenArgs&>(a) = token_args(desc, block_table, ctx_lens, q_offsets, nullptr);
  a.k = (const unsigned char*)k_pages;
  a.v = (const unsigned char*)v_pages;
  a.k_rows = (u32x4*)k_rows;
  a.v_rows = (u32x4*)v_rows;
  a.kv_heads = desc->kv_heads;
  const int64_t chunks = chunks_of(desc, 2 * (int64_t)desc->kv_heads, kFp4Loads);
  TokenGrid grid;
  if (!grid_of(desc, chunks, desc->num_tokens >= kManyTokens ? kFp4Waves : kWaves, &grid)) return SPAN_ERR_SHAPE;
  a.chunks = (int32_t)chunks;
  const bool d128 = desc->head_dim == 128;
  hipStream_t stream = (hipStream_t)desc->stream;
  auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid.grid, grid.block, 0, stream, a); };
  switch (desc->dtype) {
    case SPAN_F32:
      d128 ? start(read_kernel<F32, 128>) : start(read_kernel<F32, 64>);
      break;
    case SPAN_F16:
      d128 ? start(read_kernel<F16, 128>) : start(read_kernel<F16, 64>);
      break;
    default:
      d128 ? start(read_kernel<BF16, 128>) : start(read_kernel<BF16, 64>);
  }
  return launched();
}
