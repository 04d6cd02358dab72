// Attention of many new tokens per sequence over a cache in pages: causal, with an optional window and sinks, on the matrix cores.
//
// A workgroup of 4 wavefronts takes a tile of up to 128 query rows of one KV head - the rows are (token, query head of the group), so the heads
// that share K and V share a pass over them - and walks the cache in tiles of 64 positions (32 of fp32 rows).  Lane (c, h) = (lane % 32, lane / 32)
// plays row / column c and contraction half h of the 32x32 MFMAs; a wave has 32 query rows, which are columns throughout:
//   * scores S^T = K Q^T: Q stays in registers, K comes from LDS.  Lane (c, h) ends up with the scores of query c against positions
//     8 (r / 4) + 4 h + r % 4 of each 32, r = 0 .. 15, so a maximum or a sum is the lane's own but for one exchange of halves;
//   * outputs O^T = V^T P^T: the contraction may take the positions in any order as long as both operands do.  The order is the one the scores
//     lie in, so weights go from the registers that hold them straight into the operand; V is laid down in LDS transposed, with
//     the positions of 16 in that order, and is read like K.
// The next tile's rows are on their way to registers while this one is computed, and go to the other half of LDS after it: one barrier per tile.
// A row of K or V past the sequence's length is not read (the buffer descriptor of a page ends there) and counts as zeros.
//
// What bounds it: the matrix cores and, between their runs, the vector instructions of the softmax - a wave's own do not run beside its products, only the other
// wave's of its SIMD do.  One prompt of 8192 tokens, 32 query heads on 8 KV heads of 128, bf16: 597 us, 920 TFLOP/s of the 1208 that a product of 8192^3 reaches
// here; six chunks with a window of 1024, fp16: 186 us, 643 TFLOP/s (18 tiles a workgroup, of which 4 are cut by the window, the sinks or the diagonal).
// Tried and slower (us of those two, against 602 / 201 then): 16 query rows a wave and twice the waves 677 / 222 (twice the reads of LDS); a half tile's softmax among
// the other half's products in one wave 661 / 223; 256 rows a workgroup whose two halves take turns 575 / 231 (faster long, slower where tiles are cut).
#include "paged_device.h"

namespace spanattn {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kPromptWaves = 4, kPromptThreads = 64 * kPromptWaves;
constexpr int kPromptRows = kPromptTileRows;
static_assert(kPromptRows == 32 * kPromptWaves, "32 query rows a wave");

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  const int32_t* block_table;
  const int32_t* ctx_lens;
  const int32_t* q_offsets;
  float* part_ml;   // [slots, kPromptRows, 2]; slot = (tile * kv_heads + head) * splits + split
  float* part_acc;  // [slots, kPromptRows, D]
  int32_t batch, kv_heads, group, table_pages, page_shift, num_pages, num_tokens, max_len;
  int32_t tokens;   // of a tile: kPromptRows / group
  int32_t tiles;    // grid.y
  int32_t splits;   // workgroups that share a tile's positions
  int32_t window, sinks;  // window 0: none
  float scale_log2e;
};

template <class Elt, int D>
struct PromptShape {
  static constexpr bool kHalf = Elt::kBytes == 2;
  static constexpr int kRowBytes = D * Elt::kBytes;
  static constexpr int KT = kHalf ? 64 : 32;     // positions of a tile
  static constexpr int NB = KT / 32;
  static constexpr int NP = kRowBytes / 32;      // 16-byte pieces of a row per lane: 2 mm + h
  static constexpr int kRowsPerWave = KT / kPromptWaves;
  static constexpr int kLoads = kRowsPerWave * kRowBytes / 1024;  // 16-byte loads per lane of K (and of V) for a tile
  static constexpr int kKRow = kRowBytes + 16;
  // 16 bits: a row per dimension, 16-byte pieces of 8 positions, piece p of dimension d at p ^ (d / 16 % 8): 16 lanes that read a piece of 16 rows, or
  // write 8 bytes of it each for 16 units of dimensions, then meet in no bank twice.  (The 32 lanes of two quads that write side by side do, two and two: a third of the
  // cycles that the LDS works in a long prompt are still conflicts, 51.5 of 156 million.)  fp32: a row per position, rows 4 apart half the banks apart
  static constexpr int kVRow = kHalf ? KT * 2 + 16 : kRowBytes + 32;
  static constexpr int kKBytes = KT * kKRow, kVBytes = kHalf ? D * kVRow : KT * kVRow;
};

struct TileName {
  int b, first, tokens, pos;  // sequence; first row of q, tokens, position of the first
  int len;                    // positions that the table has
};

// Tile y: sequences in order, each in tiles of `a.tokens` tokens from its last token back (the tiles with most positions start first).
__device__ __forceinline__ TileName locate_tile(const PromptArgs& a, int y, int lane) {
  TileName t = {-1, 0, 0, 0, 0};
  int before = 0;
  for (int c = 0; c < a.batch; c += 64) {
    int begin = 0, count = 0, len = 0;
    if (c + lane < a.batch) {
      begin = clampi(a.q_offsets[c + lane], 0, a.num_tokens);
      count = clampi(a.q_offsets[c + lane + 1], begin, a.num_tokens) - begin;
      len = max(a.ctx_lens[c + lane], 0);
    }
    const int tiles = (int)((uint32_t)(count + a.tokens - 1) / (uint32_t)a.tokens);
    const int incl = before + wave_inclusive_scan(tiles);
    const uint64_t past = __builtin_amdgcn_ballot_w64(incl > y);
    if (past != 0) {
      const int at = (int)__builtin_ctzll(past);
      const int all = __builtin_amdgcn_readlane(count, at);
      const int back = y - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(tiles, at));  // tile, from the last
      const int index = __builtin_amdgcn_readlane(tiles, at) - 1 - back;
      t.b = c + at;
      const int end = __builtin_amdgcn_readlane(len, at);  // tokens keep their positions where the table ends before them
      t.len = min(end, a.max_len);
      t.first = __builtin_amdgcn_readlane(begin, at) + index * a.tokens;
      t.tokens = min(a.tokens, all - index * a.tokens);
      t.pos = end - all + index * a.tokens;
      break;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  return t;
}

// Storage type specifics of the 32x32 products.
template <class Elt>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (std::is_same<Elt, F16>::value) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
}
template <class Elt>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (std::is_same<Elt, F16>::value) return __builtin_bit_cast(uint32_t, f16x2{(_Float16)x, (_Float16)y});
  else return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// How the scheduler is to place a run of kReads reads of LDS and the kPer products that each feeds: kAhead reads first, then a read behind every kPer products.  Left
// to itself it reads two pieces, waits for both and multiplies: a trip to LDS (over 100 cycles) for every 64 cycles of products.
template <int kReads, int kPer, int kAhead>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kProducts = 0x008, kLdsReads = 0x100;
  __builtin_amdgcn_sched_group_barrier(kLdsReads, kAhead, 0);
#pragma unroll
  for (int i = 0; i < kReads - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kProducts, kPer, 0);
    __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kProducts, kAhead * kPer, 0);
}

// sum + the two values of a pair.
template <class Elt>
__device__ __forceinline__ float add_pair(uint32_t pair, float sum) {
  if constexpr (std::is_same<Elt, F16>::value) return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
  else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}

template <class Elt, int D>
__global__ __launch_bounds__(kPromptThreads)
__attribute__((amdgpu_waves_per_eu(2, 2))) void prompt_kernel(const PromptArgs a) {
  using Shape = PromptShape<Elt, D>;
  constexpr bool kHalf = Shape::kHalf;
  constexpr int KT = Shape::KT, NB = Shape::NB, NP = Shape::NP, NL = Shape::kLoads, RW = Shape::kRowsPerWave;
  constexpr int ROWB = Shape::kRowBytes, kKRow = Shape::kKRow, kVRow = Shape::kVRow;
  constexpr int kLanes = ROWB / 16;               // lanes of a row in a load of K
  constexpr int kBlocks = D / 32;
  constexpr int kAhead = 4;                       // pieces read from LDS ahead of the products they feed
  constexpr int kUnit = kHalf ? D / 16 : 4;       // 16 bits: dimensions of V that a lane transposes (of 4 positions)

  __shared__ __attribute__((aligned(16))) unsigned char s_k[2][Shape::kKBytes];
  __shared__ __attribute__((aligned(16))) unsigned char s_v[2][Shape::kVBytes];
  __shared__ uint32_t s_out[2];       // 8 bits per wave: its rows of the tile lie in a page outside the pool
  __shared__ uint32_t s_wild[2][2];   // checked pass: positions of the tile whose V row is not finite

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int h = blockIdx.x, split = blockIdx.z;
  const int group = a.group;

  const TileName t = locate_tile(a, (int)blockIdx.y, lane);
  if (t.b < 0) return;  // (the grid holds the most tiles that any offsets give)
  const int32_t* table = a.block_table + (size_t)t.b * a.table_pages;

  // This lane's query row: token `tok` of the tile, at position `at`.
  const int rows = t.tokens * group;
  const int my_row = 32 * wave + col;
  const int tok = min((int)((uint32_t)my_row / (uint32_t)group), t.tokens - 1);
  const int at = t.pos + tok, top = min(at, t.len - 1);  // its position, and the last that it may see
  auto query_row = [&](int row) {  // row (< rows) of the tile in q and out, in rows of D
    const uint32_t tk = (uint32_t)row / (uint32_t)group;
    return ((size_t)t.first + tk) * (size_t)(a.kv_heads * group) + (size_t)(h * group) + (size_t)((uint32_t)row - tk * (uint32_t)group);
  };
  const float post = Elt::post_scale(a.scale_log2e);
  constexpr float kShift = std::is_same<Elt, F16>::value ? 15.f : 0.f;  // weights times 2^15: fp16 then holds them down to 2^-39 of the heaviest

  // Positions the tile's tokens see together: [0, sinks) and [low, high).  Cache tiles: the sinks' first, then the others.
  const int high = min(t.pos + t.tokens, t.len);
  const int window = t.pos + t.tokens > a.window ? a.window : 0;  // 0: it hides nothing from any of them
  const int low = window > 0 ? max(t.pos - window + 1, 0) : 0;
  const int sinks = min(a.sinks, low);
  const int sink_tiles = (sinks + KT - 1) / KT;
  const int from = max(low / KT, sink_tiles), to = max((max(high, 0) + KT - 1) / KT, from);
  const int all_tiles = high > 0 ? sink_tiles + to - from : 0;
  const int per = (all_tiles + a.splits - 1) / a.splits;
  const int first_tile = min(split * per, all_tiles), last_tile = min(first_tile + per, all_tiles);
  auto tile_pos = [&](int i) { return (i < sink_tiles ? i : i - sink_tiles + from) * KT; };

  // The wave's tokens: what decides whether it has to mask a tile, or has nothing to do with it.
  const int wave_tok0 = (int)((uint32_t)(32 * wave) / (uint32_t)group);
  const int wave_first = t.pos + min(wave_tok0, t.tokens - 1);
  const int wave_last = t.pos + min((int)((uint32_t)(32 * wave + 31) / (uint32_t)group), t.tokens - 1);
  const bool wave_works = 32 * wave < rows;

  // ---- the cache's rows: global memory -> registers -> LDS -------------------------------------------------
  u32x4 kx[NL], vx[NL];
  uint32_t outside;
  int pages = -1;  // lane l: the page of the wave's rows of tile 64 k + l, k the last that was looked up
  const int origin = min(first_tile, max(all_tiles - 1, 0));  // the first tile, or some tile of a share without any
  auto look_up = [&](int i) {
    const int entry = (tile_pos(max(min(i + lane, last_tile - 1), 0)) + wave * RW) >> a.page_shift;
    pages = entry < a.table_pages ? table[entry] : -1;
  };
  auto fetch_rows = [&](int i) {
    const int p = tile_pos(i) + wave * RW;  // the wave's rows of the tile lie in one page
    const int entry = p >> a.page_shift, in_page = p & ((1 << a.page_shift) - 1);
    const int page = __builtin_amdgcn_readlane(pages, (i - origin) % 64);
    const bool good = (uint32_t)page < (uint32_t)a.num_pages;
    outside = !good && p < high ? 1u : 0u;
    const int there = good ? clampi(t.len - (entry << a.page_shift), 0, 1 << a.page_shift) : 0;  // rows of the page that are the sequence's
    const size_t slab = (((size_t)(good ? page : 0) * (size_t)a.kv_heads + (size_t)h) << a.page_shift) * (size_t)ROWB;
    const __amdgpu_buffer_rsrc_t kp = slab_resource((const char*)a.k + slab, (uint32_t)(there * ROWB));
    const __amdgpu_buffer_rsrc_t vp = slab_resource((const char*)a.v + slab, (uint32_t)(there * ROWB));
    const uint32_t base = (uint32_t)in_page * ROWB;
#pragma unroll
    for (int i = 0; i < NL; ++i) kx[i] = __builtin_amdgcn_raw_buffer_load_b128(kp, base + 16u * (uint32_t)lane + 1024u * i, 0, 0);
    if constexpr (kHalf) {
      // lane: positions 4 (lane / 16) + i of the wave's 16, dimensions kUnit (lane % 16) on
      const uint32_t vat = base + (uint32_t)(4 * (lane >> 4)) * ROWB + (uint32_t)(lane & 15) * (kUnit * 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kUnit == 8) vx[i] = __builtin_amdgcn_raw_buffer_load_b128(vp, vat + (uint32_t)i * ROWB, 0, 0);
        else {
          const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(vp, vat + (uint32_t)i * ROWB, 0, 0);
          vx[i / 2][2 * (i & 1)] = w[0];
          vx[i / 2][2 * (i & 1) + 1] = w[1];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) vx[i] = __builtin_amdgcn_raw_buffer_load_b128(vp, base + 16u * (uint32_t)lane + 1024u * i, 0, 0);
    }
  };
  auto fetch = [&](int i) {
    if (i > origin && (i - origin) % 64 == 0) look_up(i);
    fetch_rows(i);
  };
  // Pages and queries are on their way together, then the first rows; only then are the queries waited for.
  look_up(origin);
  u32x4 qr[NP];
  {
    const char* src = (const char*)a.q + query_row(min(my_row, rows - 1)) * (size_t)ROWB + 16 * half;
#pragma unroll
    for (int mm = 0; mm < NP; ++mm) qr[mm] = *reinterpret_cast<const u32x4*>(src + 32 * mm);
  }
  fetch_rows(origin);
#pragma unroll
  for (int mm = 0; mm < NP; ++mm) {
#pragma unroll
    for (int k = 0; k < 4; ++k) qr[mm][k] = Elt::scale_query(qr[mm][k], a.scale_log2e);
  }
  auto lay_down = [&](int buf, auto checked) {
    constexpr bool kChecked = decltype(checked)::value;
    if (lane == 0) reinterpret_cast<unsigned char*>(&s_out[buf])[wave] = (unsigned char)outside;
    unsigned char* kd = &s_k[buf][(wave * RW + lane / kLanes) * kKRow + 16 * (lane % kLanes)];
#pragma unroll
    for (int i = 0; i < NL; ++i) *reinterpret_cast<u32x4*>(kd + i * (64 / kLanes) * kKRow) = kx[i];
    if constexpr (kHalf) {
      constexpr int W = kUnit / 2;  // dwords of a position
      uint32_t x[4][W];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int k = 0; k < W; ++k) x[i][k] = kUnit == 8 ? vx[i][k] : vx[i / 2][2 * (i & 1) + k];
      }
      const int quad = lane >> 4;  // positions 16 wave + 4 quad ..
      if constexpr (kChecked) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bool wild = false;
#pragma unroll
          for (int k = 0; k < W; ++k) {
            const uint32_t w = x[i][k];
            const bool lo = Elt::not_finite(w & 0xffffu), hi = Elt::not_finite(w & 0xffff0000u);
            wild = wild || lo || hi;
            x[i][k] = (lo ? 0u : w & 0xffffu) | (hi ? 0u : w & 0xffff0000u);
          }
          if (wild) atomicOr(&s_wild[buf][wave / 2], 1u << (16 * (wave & 1) + 4 * quad + i));
        }
      }
      // piece of 8 positions: 0-3 and 8-11 of the wave's 16 (quads 0, 2), or 4-7 and 12-15 (quads 1, 3)
      const int piece = 2 * wave + (quad & 1), within = 8 * (quad >> 1);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const int d = kUnit * (lane & 15) + j;
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        const u32x2 w = {__builtin_amdgcn_perm(x[1][j / 2], x[0][j / 2], sel), __builtin_amdgcn_perm(x[3][j / 2], x[2][j / 2], sel)};
        *reinterpret_cast<u32x2*>(&s_v[buf][d * kVRow + 16 * (piece ^ ((d >> 4) & 7)) + within]) = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = wave * RW + i * (64 / kLanes) + lane / kLanes;
        u32x4 w = vx[i];
        if constexpr (kChecked) {
          bool wild = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            wild = wild || Elt::not_finite(w[k]);
            w[k] = Elt::not_finite(w[k]) ? 0u : w[k];
          }
          if (wild) atomicOr(&s_wild[buf][0], 1u << row);
        }
        *reinterpret_cast<u32x4*>(&s_v[buf][row * kVRow + 16 * (lane % kLanes)]) = w;
      }
    }
  };

  constexpr float kLargeShift = 4194304.f;  // 2^22: a rounding of a quarter at most
  float shift = kShift;
  bool large = false;
  float ref = -INFINITY, lsum = 0.f;  // reference of the weights: the largest unscaled score; this lane's share of their sum
  f32x16 O[kBlocks];
  // A weight is exp2(score * post + shift), shift = kShift - reference * post rounded.  What the rounding leaves is a factor exp2(slack) of all weights of one
  // reference: it goes out with their sum, but where the reference moves or shares are joined it has to be taken into account (without that, fp32 scores near 2^13 that
  // lie close to one another gave outputs off by 3e-5, near 2^21 by 7e-3).
  float slack = 0.f;
  auto sees = [&](int p) { return p <= top && (window == 0 || p > at - window || p < a.sinks); };

  const int v_lane = col * kVRow + 16 * (half ^ (col >> 4));
  auto compute = [&](int buf, int p0, auto checked) {
    constexpr bool kChecked = decltype(checked)::value;
    if (!wave_works || p0 > wave_last) return;
    if (window > 0 && p0 + KT - 1 <= wave_first - window && p0 >= a.sinks) return;
    constexpr f32x16 kZero = {};
    f32x16 S[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const unsigned char* kr = &s_k[buf][(32 * n + col) * kKRow + 16 * half];
#pragma unroll
      for (int mm = 0; mm < NP; ++mm) {
        const u32x4 km = *reinterpret_cast<const u32x4*>(kr + 32 * mm);
        if constexpr (kHalf) {
          S[n] = mfma32<Elt>(km, qr[mm], mm == 0 ? kZero : S[n]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t kw = km[k], qw = qr[mm][k];
            S[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, kw), __builtin_bit_cast(float, qw), mm == 0 && k == 0 ? kZero : S[n], 0, 0, 0);
          }
        }
      }
    }
    reads_ahead<NB * NP, kHalf ? 1 : 4, kAhead>();
    const uint32_t out_bits = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_out[buf]);
    const bool whole = p0 + KT - 1 <= min(wave_first, t.len - 1) && (window == 0 || p0 > wave_last - window || p0 + KT <= a.sinks) && out_bits == 0;
    if (!whole) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        // bit i: position pn + i counts, which `sees` says
        const int pn = p0 + 32 * n;
        auto first = [](int k) { return k >= 32 ? ~0u : (1u << max(k, 0)) - 1u; };
        uint32_t bits = first(top - pn + 1);
        if (window > 0) bits &= ~first(at - window + 1 - pn) | first(a.sinks - pn);
        if constexpr (RW == 16) bits &= ~((out_bits >> (16 * n) & 1u) * 0xffffu | (out_bits >> (16 * n + 8) & 1u) * 0xffff0000u);
        else bits &= ~(out_bits * 0xffu);
        bits >>= 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) S[n][r] = (bits >> (8 * (r / 4) + r % 4) & 1u) != 0 ? S[n][r] : -INFINITY;
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, S[n][r]);
    }
    if (__builtin_amdgcn_ballot_w64(mx > ref) != 0) {
      const Swapped sw = swap_lanes<32>(mx, mx);
      const float ref_new = fmaxf(ref, fmaxf(sw.first, sw.second)), safe = ref_new == -INFINITY ? 0.f : ref_new;
      shift = kShift - safe * post;
      large = __builtin_amdgcn_ballot_w64(!(fabsf(shift) < kLargeShift)) != 0;
      const float slack_new = large ? 0.f : fmaf(safe, post, shift) - kShift;
      const float alpha = __builtin_amdgcn_exp2f(fmaf(ref - safe, post, slack_new - slack));
      ref = ref_new;
      slack = slack_new;
      lsum *= alpha;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) O[e] *= alpha;
    }
    // Where the shift's rounding is no longer small the difference from the reference is taken first, which is exact.
    if (__builtin_expect(large, 0)) {
      const float safe = ref == -INFINITY ? 0.f : ref;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[n][r] = __builtin_amdgcn_exp2f(fmaf(S[n][r] - safe, post, kShift));
      }
    } else {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[n][r] = __builtin_amdgcn_exp2f(fmaf(S[n][r], post, shift));
      }
    }
    if constexpr (kHalf) {
      // A weight meets V rounded to the storage type, once, and the sum is that of the rounded ones.  The output is rounded to the same type, so that this is the smaller of two
      // errors of a size: bf16 outputs are 0.0020 (relative) from the 64-bit ones where weights of 32 bits give 0.0015, fp16 0.00028 and 0.00021.  A second term for what the
      // rounding leaves reaches those and takes twice the products of V: a prompt of 8192 602 -> 803 us, chunks in a window of 1024 188 -> 245.
      u32x4 P[NB][2];
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            P[n][c][k] = pack2<Elt>(S[n][8 * c + 2 * k], S[n][8 * c + 2 * k + 1]);
            sum[k] = add_pair<Elt>(P[n][c][k], sum[k]);
          }
        }
      }
      lsum += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      const unsigned char* vr = &s_v[buf][0] + v_lane;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            // piece 4 n + 2 c + half of dimension 32 e + col, at its place: bit 0 of the turn is the lane's, the others are e's
            const u32x4 vm = *reinterpret_cast<const u32x4*>(vr + 32 * e * kVRow + 16 * ((4 * n + 2 * c) ^ (2 * e)));
            O[e] = mfma32<Elt>(vm, P[n][c], O[e]);
          }
        }
      }
      reads_ahead<kBlocks * NB * 2, 1, kAhead>();
    } else {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[r & 3] += S[0][r];
      lsum += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float vm = *reinterpret_cast<const float*>(&s_v[buf][(8 * (r / 4) + r % 4 + 4 * half) * kVRow + 4 * (32 * e + col)]);
          O[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(vm, S[0][r], O[e], 0, 0, 0);
        }
      }
    }
    if constexpr (kChecked) {
      // Values of V that are not finite were left out of the products; here they meet the weights of the queries that see them, and of no others
      // (0 * Inf would be NaN).
#pragma unroll 1
      for (int w = 0; w < NB; ++w) {
#pragma unroll 1
        for (uint32_t todo = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_wild[buf][w]); todo != 0; todo &= todo - 1) {
          const int i = __builtin_ctz(todo);           // position 32 w + i: scores' register 4 (i / 8) + i % 4 of half i / 4 % 2
          const int p = p0 + 32 * w + i, r_of = 4 * (i >> 3) + (i & 3);
          float x = 0.f;
#pragma unroll
          for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x = n == w && r == r_of ? S[n][r] : x;
          }
          x = __shfl(x, 32 * ((i >> 2) & 1) + col, 64);
          const int row = pool_row(table, p, a.page_shift, a.num_pages);
          if (row < 0 || !sees(p)) continue;
          const size_t page = (size_t)(row >> a.page_shift), in_page = (size_t)(row & ((1 << a.page_shift) - 1));
          const char* src = (const char*)a.v + (((page * (size_t)a.kv_heads + (size_t)h) << a.page_shift) + in_page) * (size_t)ROWB;
#pragma unroll
          for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              float vf[4];
              const char* from4 = src + (32 * e + 8 * g + 4 * half) * Elt::kBytes;
              if constexpr (kHalf) Elt::unpack4(*reinterpret_cast<const u32x2*>(from4), vf);
              else Elt::unpack4(*reinterpret_cast<const u32x4*>(from4), vf);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const bool wild = !(fabsf(vf[k]) < INFINITY);
                O[e][4 * g + k] = wild ? fmaf(x, vf[k], O[e][4 * g + k]) : O[e][4 * g + k];
              }
            }
          }
        }
      }
    }
  };

  auto walk = [&](auto checked) {
    constexpr bool kChecked = decltype(checked)::value;
    ref = -INFINITY;
    lsum = 0.f;
    shift = kShift;
    slack = 0.f;
    large = false;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
      for (int r = 0; r < 16; ++r) O[e][r] = 0.f;
    }
    if (first_tile >= last_tile) return;
    if (kChecked) {
      look_up(origin);
      fetch_rows(origin);
      if (tid < 4) s_wild[tid >> 1][tid & 1] = 0u;
      __syncthreads();
    }
    lay_down(0, checked);
    __syncthreads();
    int buf = 0;
    for (int i = first_tile; i < last_tile; ++i) {
      fetch(min(i + 1, last_tile - 1));  // (the last tile a second time rather than a branch, which would cost copies of all these registers)
      compute(buf, tile_pos(i), checked);
      if (i + 1 == last_tile) break;
      if (kChecked) {
        __syncthreads();
        if (tid < 2) s_wild[buf][tid] = 0u;  // (for the tile after next)
      }
      lay_down(buf ^ 1, checked);
      __syncthreads();
      buf ^= 1;
    }
    if (kChecked) __syncthreads();  // (as the vote does behind the other pass: nobody reads LDS any more)
  };
  walk(std::false_type{});
  {
    float z = 0.f;  // stays 0 unless some output is Inf or NaN
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
      for (int r = 0; r < 16; ++r) z = fmaf(O[e][r], 0.f, z);
    }
    if (__builtin_expect(__syncthreads_or(z != 0.f), 0)) walk(std::true_type{});
  }

  const Swapped both = swap_lanes<32>(lsum, lsum);
  lsum = both.first + both.second;
  if (a.splits > 1) {
    if (my_row < rows) {
      const float level = __builtin_amdgcn_exp2f(-slack);  // (the merge takes a share's weights relative to its reference)
      lsum *= level;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) O[e] *= level;
      const size_t slot = ((size_t)blockIdx.y * a.kv_heads + h) * (size_t)a.splits + (size_t)split;
      const size_t row = slot * kPromptRows + (size_t)my_row;
      if (half == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * row) = f32x2{ref, lsum};
      float* acc = a.part_acc + row * D + 4 * half;
#pragma unroll
      for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(acc + 32 * e + 8 * g) = f32x4{O[e][4 * g], O[e][4 * g + 1], O[e][4 * g + 2], O[e][4 * g + 3]};
      }
    }
    return;
  }
  // The wave's rows through LDS, so that they are stored whole (its own part of the first half, which nobody reads any more).
  const float inv = 1.f / (lsum != 0.f ? lsum : 1.f);
  static_assert(32 * kPromptWaves * kKRow <= 2 * Shape::kKBytes || kHalf == false, "the tile's outputs fit");
  if constexpr (kHalf) {
    unsigned char* mine = &s_k[0][0] + wave * 32 * kKRow;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const u32x2 w = {pack2<Elt>(O[e][4 * g] * inv, O[e][4 * g + 1] * inv), pack2<Elt>(O[e][4 * g + 2] * inv, O[e][4 * g + 3] * inv)};
        *reinterpret_cast<u32x2*>(mine + col * kKRow + 2 * (32 * e + 8 * g + 4 * half)) = w;
      }
    }
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < 32 * kLanes / 64; ++i) {
      const int r = i * (64 / kLanes) + lane / kLanes;
      if (32 * wave + r < rows)
        *reinterpret_cast<u32x4*>((char*)a.out + query_row(32 * wave + r) * (size_t)ROWB + 16 * (lane % kLanes)) =
            *reinterpret_cast<const u32x4*>(mine + r * kKRow + 16 * (lane % kLanes));
    }
  } else if (my_row < rows) {
    float* out = (float*)a.out + query_row(my_row) * (size_t)D + 4 * half;
#pragma unroll
    for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(out + 32 * e + 8 * g) = f32x4{O[e][4 * g] * inv, O[e][4 * g + 1] * inv, O[e][4 * g + 2] * inv, O[e][4 * g + 3] * inv};
    }
  }
}

// The states of the workgroups that shared a tile's positions become one: a thread has four columns of a row.
template <class Elt, int D>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const PromptArgs a) {
  const int lane = threadIdx.x & 63, h = blockIdx.x;
  const TileName t = locate_tile(a, (int)blockIdx.y, lane);
  if (t.b < 0) return;
  const float post = Elt::post_scale(a.scale_log2e);
  const int row = (int)(blockIdx.z * 256 + threadIdx.x) / (D / 4), column = (int)threadIdx.x % (D / 4) * 4;
  if (row >= t.tokens * a.group) return;
  const size_t slot0 = ((size_t)blockIdx.y * a.kv_heads + h) * (size_t)a.splits;
  float M = -INFINITY, L = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 8;  // states on their way at once
  for (int s0 = 0; s0 < a.splits; s0 += kAhead) {
    f32x2 ml[kAhead];
    f32x4 os[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const size_t at = (slot0 + (size_t)min(s0 + k, a.splits - 1)) * kPromptRows + (size_t)row;  // (past the end: the last once more, unused)
      ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + 2 * at);
      os[k] = *reinterpret_cast<const f32x4*>(a.part_acc + at * D + column);
    }
    const float before = M;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (s0 + k >= a.splits) ml[k][1] = 0.f;
      if (ml[k][1] != 0.f) M = fmaxf(M, ml[k][0]);  // (0: nothing seen there; a NaN sum counts)
    }
    const float safe = M == -INFINITY ? 0.f : M, old = __builtin_amdgcn_exp2f((before - safe) * post);
    L *= old;
    o *= old;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (ml[k][1] != 0.f) {
        const float w = __builtin_amdgcn_exp2f((ml[k][0] - safe) * post);
        L = fmaf(w, ml[k][1], L);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = fmaf(w, os[k][c], o[c]);
      }
    }
  }
  const float sum = L != 0.f ? L : 1.f;
  const uint32_t tk = (uint32_t)row / (uint32_t)a.group;
  const size_t to = (((size_t)t.first + tk) * (size_t)(a.kv_heads * a.group) + (size_t)(h * a.group) + (size_t)((uint32_t)row - tk * (uint32_t)a.group)) * D + column;
  if constexpr (Elt::kBytes == 2) {
    *reinterpret_cast<u32x2*>((char*)a.out + to * 2) = u32x2{pack2<Elt>(o[0] / sum, o[1] / sum), pack2<Elt>(o[2] / sum, o[3] / sum)};
  } else {
    *reinterpret_cast<f32x4*>((float*)a.out + to) = f32x4{o[0] / sum, o[1] / sum, o[2] / sum, o[3] / sum};
  }
}

template <class Elt, int D>
int run_prompt(const PromptArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((prompt_kernel<Elt, D>), dim3((unsigned)a.kv_heads, (unsigned)a.tiles, (unsigned)a.splits), dim3(kPromptThreads), 0, stream, a);
  const int rc = launched();
  if (rc != SPAN_OK || a.splits == 1) return rc;
  const unsigned z = (unsigned)(kPromptRows * (D / 4) / 256);
  hipLaunchKernelGGL((prompt_merge_kernel<Elt, D>), dim3((unsigned)a.kv_heads, (unsigned)a.tiles, z), dim3(256), 0, stream, a);
  return launched();
}

}  // namespace
}  // namespace spanattn

extern "C" int paged_prompt_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                                 const int32_t* ctx_lens, const int32_t* q_offsets, float scale, void* out) {
  using namespace spanattn;
  const int rc = check_paged(desc);
  if (rc != SPAN_OK) return rc;
  if (!block_table || !ctx_lens || !q_offsets || !k_pages || !v_pages) return SPAN_ERR_NULL;
  if (desc->num_tokens == 0) return SPAN_OK;
  if (!q || !out) return SPAN_ERR_NULL;
  const PromptPlan p = plan_prompt(desc);
  if (p.tiles > 65535) return SPAN_ERR_SHAPE;
  const size_t need = prompt_workspace(desc, p);
  if (need > 0 && (!desc->workspace || ((uintptr_t)desc->workspace & 255u) || desc->workspace_bytes < need)) return SPAN_ERR_WORKSPACE;
  PromptArgs a;
  a.q = q;
  a.k = k_pages;
  a.v = v_pages;
  a.out = out;
  a.block_table = block_table;
  a.ctx_lens = ctx_lens;
  a.q_offsets = q_offsets;
  a.part_ml = need ? (float*)desc->workspace : nullptr;
  a.part_acc = need ? (float*)((char*)desc->workspace + p.acc) : nullptr;
  a.batch = desc->batch;
  a.kv_heads = desc->kv_heads;
  a.group = desc->heads / desc->kv_heads;
  a.table_pages = desc->table_pages;
  a.page_shift = page_shift(desc);
  a.num_pages = desc->num_pages;
  a.num_tokens = desc->num_tokens;
  a.max_len = capacity(desc);
  a.tokens = p.tokens;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.window = desc->window;
  a.sinks = desc->sinks < a.max_len ? desc->sinks : a.max_len;
  a.scale_log2e = scale * 1.4426950408889634f;
  hipStream_t stream = (hipStream_t)desc->stream;
  const bool d128 = desc->head_dim == 128;
  switch (desc->dtype) {
    case SPAN_F32: return d128 ? run_prompt<F32, 128>(a, stream) : run_prompt<F32, 64>(a, stream);
    case SPAN_F16: return d128 ? run_prompt<F16, 128>(a, stream) : run_prompt<F16, 64>(a, stream);
    default: return d128 ? run_prompt<BF16, 128>(a, stream) : run_prompt<BF16, 64>(a, stream);
  }
}
