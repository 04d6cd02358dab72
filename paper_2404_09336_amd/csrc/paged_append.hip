// New rows into the pages with K (and q) turned by the angles of their positions, as they are or in 4 bits, and rows of 4-bit pages back as values.
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
  int32_t kv_chunks, q_chunks;   // waves that a token's rows of K (as many of V), and of q, take
};

struct ReadArgs : TokenArgs {
  const unsigned char* k;
  const unsigned char* v;
  u32x4* k_rows;
  u32x4* v_rows;
  int32_t kv_heads, kv_chunks;
};

constexpr int kTurnLoads = 4;  // pieces of 16 bytes per lane
constexpr int kTurnPieces = 64 * kTurnLoads;

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
  int partner;  // halves: pieces from a lane's to that of the other channels
  bool turned;

  __device__ __forceinline__ void load(const TurnArgs& a, int position, int piece) {
    const int d = piece * kPer, half = a.channels / 2;
    turned = d < a.channels;
    if (!turned) return;
    const bool second = !kPaired && d >= half;
    const int first = kPaired ? d / 2 : d - (second ? half : 0);
    partner = (second ? -half : half) / kPer;
    const bool known = (uint32_t)position < (uint32_t)a.angle_rows;
    const float* row = a.angles + (size_t)(known ? position : 0) * (size_t)a.channels + first;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      cosine[i] = known ? row[i] : NAN;
      sine[i] = known ? (second || kPaired ? row[half + i] : -row[half + i]) : NAN;
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

// x to fp32, inexact values to the neighbour with an odd last bit: rounded again to fewer bits, with ties to even, it becomes what x would.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double back = (double)f;
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (fabs(back) > fabs(x)) u -= 1u;
  if (back != x) u |= 1u;
  return __builtin_bit_cast(float, u);
}
// The same as turn, to the odd neighbour of the exact value: products of two fp32 are exact in 64 bits, their sum is rounded once.
template <class Elt, bool kPaired>
__device__ __forceinline__ void turn_exactly(const Angles<Elt, kPaired>& g, float* x, const float* other) {
#pragma unroll
  for (int i = 0; i < Elt::kPerVec; ++i) {
    if constexpr (kPaired) {
      if (i & 1) continue;
      const double one = x[i], two = x[i + 1], c = g.cosine[i / 2], s = g.sine[i / 2];
      x[i] = to_odd(fma(one, c, -(two * s)));
      x[i + 1] = to_odd(fma(one, s, two * c));
    } else {
      x[i] = to_odd(fma((double)x[i], (double)g.cosine[i], (double)other[i] * (double)g.sine[i]));
    }
  }
}

// Exponent byte of the block of 32 channels that kLanes lanes hold together, by the largest magnitude (as bits: NaN above infinity above numbers).
template <int kPer>
__device__ __forceinline__ uint32_t block_exponent(const float* x) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) most = max(most, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
  most = max(most, (uint32_t)dpp_i<0xB1>((int)most));            // quad_perm [1,0,3,2]
  most = max(most, (uint32_t)dpp_i<0x4E>((int)most));            // quad_perm [2,3,0,1]
  if (kPer == 4) most = max(most, (uint32_t)dpp_i<0x141>((int)most));  // row_half_mirror
  constexpr uint32_t kSeven = 0x00600000u;                       // mantissa of 7 = 1.75 * 2^2
  constexpr uint32_t kMost = ((uint32_t)(kFp4MostExponent + 2 + 127) << 23) | kSeven;
  if (most > kMost) return 255u;
  const int e = (int)(most >> 23) - 2 + ((most & 0x7fffffu) > kSeven ? 1 : 0);  // e + 127
  return (uint32_t)max(e, kFp4LeastExponent + 127);
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

// A wave takes up to 4 KB of one token's rows of K, of V, or of q.  Bound by memory where there are many rows, by the chain of trips (offsets, length, page) where there are few.
template <class Elt, int D, bool kFp4, bool kPaired>
__global__ __launch_bounds__(256) void turn_kernel(const TurnArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;  // pieces of a row
  const int lane = threadIdx.x & 63;
  const uint32_t unit = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4u + (threadIdx.x >> 6)));
  const uint32_t chunks = 2u * (uint32_t)a.kv_chunks + (uint32_t)a.q_chunks;
  const int t = (int)(unit / chunks);
  int c = (int)(unit % chunks);
  if (t >= a.num_tokens) return;
  const bool is_k = c < a.kv_chunks, is_v = !is_k && c < 2 * a.kv_chunks;
  c -= is_k ? 0 : is_v ? a.kv_chunks : 2 * a.kv_chunks;
  const int pieces = (is_k || is_v ? a.kv_heads : a.heads) * kRow;
  const u32x4* from = (is_k ? a.k_new : is_v ? a.v_new : a.q) + (size_t)t * pieces;
  const int first = c * kTurnPieces + lane, piece = first % kRow;
  u32x4 x[kTurnLoads], other[kTurnLoads];
#pragma unroll
  for (int i = 0; i < kTurnLoads; ++i) x[i] = from[min(first + 64 * i, pieces - 1)];
  const bool turns = !is_v && a.channels > 0;
  const Token tok = find_token(a, t, lane);
  if (tok.b < 0) return;
  Angles<Elt, kPaired> g;
  g.turned = false;
  g.partner = 0;
  if (turns) g.load(a, tok.position, piece);
  if (!kPaired && turns) {
#pragma unroll
    for (int i = 0; i < kTurnLoads; ++i) {
      const int at = min(first + 64 * i, pieces - 1);
      other[i] = from[g.turned && first + 64 * i < pieces ? at + g.partner : at];
    }
  }
  if (is_k && c == 0 && a.positions != nullptr && (uint32_t)tok.p < (uint32_t)a.max_len) {
    for (int h = lane; h < a.kv_heads; h += 64) a.positions[((size_t)tok.b * a.kv_heads + h) * (size_t)a.max_len + tok.p] = tok.position;
  }
  int row = -1;
  if (is_k || is_v) {
    row = token_row(a, tok);
    if (row < 0) return;
  }
  const size_t page = (size_t)(max(row, 0) >> a.page_shift);
  const uint32_t page_rows = 1u << a.page_shift, in_page = (uint32_t)max(row, 0) & (page_rows - 1u);
#pragma unroll
  for (int i = 0; i < kTurnLoads; ++i) {
    const int at = first + 64 * i;
    float f[kPer];
    const bool to_fp4 = kFp4 && (is_k || is_v);
    if (to_fp4 || g.turned) {
      Elt::unpack(x[i], f);
      if (g.turned) {
        float o[kPer];
        if constexpr (!kPaired) Elt::unpack(other[i], o);
        if (to_fp4) turn_exactly<Elt, kPaired>(g, f, o);
        else turn<Elt, kPaired>(g, f, o);
        if (!to_fp4) x[i] = pack_values<Elt>(f);
      }
    }
    if constexpr (kFp4) {
      if (is_k || is_v) {  // (all lanes: a block's are exchanged; the rows of one token end with a whole block)
        const uint32_t exponent = block_exponent<kPer>(f), w = to_codes<kPer>(f, exponent);
        if (at < pieces) {
          const int h = at / kRow;
          const uint32_t ch = (uint32_t)piece * kPer;
          unsigned char* to = (unsigned char*)(is_k ? a.k : a.v) + (page * (size_t)a.kv_heads + (size_t)h) * ((size_t)page_rows * (D / 2 + D / kFp4Block));
          if (is_k) {
            if constexpr (kPer == 8) *(uint32_t*)(to + code_at<D, false>(in_page, ch)) = w;
            else *(uint16_t*)(to + code_at<D, false>(in_page, ch)) = (uint16_t)w;
          } else if constexpr (kPer == 8 && D == 128) {
            *(uint32_t*)(to + code_at<D, true>(in_page, ch)) = w;
          } else {
            *(uint16_t*)(to + code_at<D, true>(in_page, ch)) = (uint16_t)w;
            if constexpr (kPer == 8) *(uint16_t*)(to + code_at<D, true>(in_page, ch + 4u)) = (uint16_t)(w >> 16);
          }
          if (ch % kFp4Block == 0) to[exponent_at<D>(page_rows, in_page, ch)] = (unsigned char)exponent;
        }
        continue;
      }
    }
    if (at < pieces) {
      if (is_k || is_v) {
        const size_t to = (((page * (size_t)a.kv_heads + (size_t)(at / kRow)) << a.page_shift) + in_page) * (size_t)kRow + (size_t)piece;
        ((u32x4*)(is_k ? a.k : a.v))[to] = x[i];
      } else {
        a.q_out[(size_t)t * pieces + at] = x[i];
      }
    }
  }
}

template <class Elt, int D>
__global__ __launch_bounds__(256) void read_kernel(const ReadArgs a) {
  constexpr int kPer = Elt::kPerVec, kRow = D / kPer;
  const int lane = threadIdx.x & 63;
  const uint32_t unit = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4u + (threadIdx.x >> 6)));
  const uint32_t chunks = 2u * (uint32_t)a.kv_chunks;
  const int t = (int)(unit / chunks);
  int c = (int)(unit % chunks);
  if (t >= a.num_tokens) return;
  const bool is_k = c < a.kv_chunks;
  if (!is_k) c -= a.kv_chunks;
  const Token tok = find_token(a, t, lane);
  if (tok.b < 0) return;
  const int row = token_row(a, tok);
  if (row < 0) return;
  const size_t page = (size_t)(row >> a.page_shift);
  const uint32_t page_rows = 1u << a.page_shift, in_page = (uint32_t)row & (page_rows - 1u);
  const int pieces = a.kv_heads * kRow;
#pragma unroll
  for (int i = 0; i < kTurnLoads; ++i) {
    const int at = c * kTurnPieces + lane + 64 * i;
    if (at >= pieces) continue;
    const uint32_t ch = (uint32_t)(at % kRow) * kPer;
    const unsigned char* of = (is_k ? a.k : a.v) + (page * (size_t)a.kv_heads + (size_t)(at / kRow)) * ((size_t)page_rows * (D / 2 + D / kFp4Block));
    const float scale = __builtin_bit_cast(float, (uint32_t)of[exponent_at<D>(page_rows, in_page, ch)] << 23);
    uint32_t w;
    if (is_k) w = kPer == 8 ? *(const uint32_t*)(of + code_at<D, false>(in_page, ch)) : (uint32_t) * (const uint16_t*)(of + code_at<D, false>(in_page, ch));
    else if constexpr (kPer == 8 && D == 128) w = *(const uint32_t*)(of + code_at<D, true>(in_page, ch));
    else {
      w = *(const uint16_t*)(of + code_at<D, true>(in_page, ch));
      if constexpr (kPer == 8) w |= (uint32_t) * (const uint16_t*)(of + code_at<D, true>(in_page, ch + 4u)) << 16;
    }
    float f[8];
    f32x2 two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    f[0] = two[0], f[1] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    f[2] = two[0], f[3] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    f[4] = two[0], f[5] = two[1];
    two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    f[6] = two[0], f[7] = two[1];
    (is_k ? a.k_rows : a.v_rows)[(size_t)t * pieces + at] = pack_values<Elt>(f);
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

int32_t chunks_of(const span_paged_desc_t* d, int32_t heads) {
  const int64_t pieces = (int64_t)heads * (d->head_dim * (d->dtype == SPAN_F32 ? 4 : 2) / 16);
  return (int32_t)((pieces + kTurnPieces - 1) / kTurnPieces);
}

// Workgroups of four waves, one wave for each of so many chunks of a token; false: more than a grid holds.
bool grid_of(const span_paged_desc_t* d, int64_t chunks, dim3* grid) {
  const int64_t waves = (int64_t)d->num_tokens * chunks;
  if (waves > 0x7fffffff) return false;
  *grid = dim3((unsigned)((waves + 3) / 4));
  return true;
}

template <class Elt, int D, bool kFp4>
void start_turn(const TurnArgs& a, bool paired, dim3 grid, hipStream_t stream) {
  if (paired) hipLaunchKernelGGL((turn_kernel<Elt, D, kFp4, true>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((turn_kernel<Elt, D, kFp4, false>), grid, dim3(256), 0, stream, a);
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
  if (q && !rotation) return SPAN_ERR_SHAPE;
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
  a.kv_chunks = chunks_of(d, d->kv_heads);
  a.q_chunks = q ? chunks_of(d, d->heads) : 0;
  dim3 grid;
  if (!grid_of(d, 2 * (int64_t)a.kv_chunks + a.q_chunks, &grid)) return SPAN_ERR_SHAPE;
  const bool paired = rotation && rotation->paired, d128 = d->head_dim == 128;
  hipStream_t stream = (hipStream_t)d->stream;
  switch (d->dtype) {
    case SPAN_F32:
      d128 ? start_turn<F32, 128, kFp4>(a, paired, grid, stream) : start_turn<F32, 64, kFp4>(a, paired, grid, stream);
      break;
    case SPAN_F16:
      d128 ? start_turn<F16, 128, kFp4>(a, paired, grid, stream) : start_turn<F16, 64, kFp4>(a, paired, grid, stream);
      break;
    default:
      d128 ? start_turn<BF16, 128, kFp4>(a, paired, grid, stream) : start_turn<BF16, 64, kFp4>(a, paired, grid, stream);
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
  a.kv_chunks = chunks_of(desc, desc->kv_heads);
  dim3 grid;
  if (!grid_of(desc, 2 * (int64_t)a.kv_chunks, &grid)) return SPAN_ERR_SHAPE;
  const bool d128 = desc->head_dim == 128;
  hipStream_t stream = (hipStream_t)desc->stream;
  auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a); };
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
