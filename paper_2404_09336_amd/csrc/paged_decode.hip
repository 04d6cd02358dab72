// One-token attention over a cache in pages, for up to 16 query heads per KV head.
//
// A workgroup of 4 wavefronts takes one slice of a (sequence, KV head) pair's positions and all query heads of the group, which
// are the query columns of 16x16 MFMAs: the products, the storage types' weights and the hand-over between slices are those of
// the few-query kernel (span_matrix.hip), with heads in place of tokens.  What differs:
//   * A row's address comes from the block table.  A wave tabulates the pool rows of its next 512 positions in LDS (one load of
//     the table per row, coalesced where positions follow one another), so that the row loads do not wait for the table one by one.
//   * Every query column sees the same rows, so there is no mask but for rows past the slice's end and of pages outside the pool.
//   * The slices are found on the device from the lengths themselves (locate_slice): a captured call stays level when lengths grow.
//   * Weights per position (for an eviction) need the final maxima and sums: the scores go to the workspace as they are taken and a
//     second kernel turns them into weights, 4 bytes a score against the 2 * head_dim * element bytes of a row.  Where no sequence is cut
//     and the positions are few (kPagedOwnWeights) the workgroup does that itself.
// What bounds it: memory, and for short calls the chain of trips before the first rows and of the hand-over behind the last.  64 sequences
// of 512 .. 4096 positions, 32 query heads on 8 KV heads of 128, bf16: 104 us, 6.0 TB/s; a window of 1024 over 32 of them, fp16: 26.7 us,
// 5.0 TB/s; 4 of 8000 .. 32768: 55.9 us, 5.6 TB/s, with weights 69 (the scores' 10 MB cost 8 us on their way out and 5.4 in the second
// launch; stored through or past the caches they cost 4 to 7 us more); one sequence of 256 positions, fp32: 8.0 us.
#include "paged_attend.h"

namespace spanattn {

namespace {

constexpr int kPWin = 512;  // rows of a wave whose pool rows are tabulated at a time

template <class Elt, int D>
struct PagedShape {
  static constexpr int kRowBytes = D * Elt::kBytes;
  static constexpr int NK = kRowBytes / 64;        // 16-byte pieces of a K row per lane
  static constexpr int NE = D / 16;                // values of a V row per lane
  static constexpr int VW = NE * Elt::kBytes / 4;  // dwords they fill: 2, 4, or 8 (fp32, D = 128: two pieces)
  // Groups of 16 rows in a step.  More of them, with fewer waves (two of 256-byte rows at three per SIMD, four at two), are slower: a call of few
  // positions by its longer code, one of many by the waves (31 drawn and listed calls, mean 12.2 us -> 12.9 and 14.4).
  static constexpr int S = kRowBytes == 128 ? 2 : 1;
  static constexpr int kWaves = kRowBytes == 512 ? 2 : 4;  // per SIMD
};

// weights[b, h, p] += sum over the group's heads of exp2((score - maximum) * post) / sum, for the positions with virtual numbers v0 .. v0 + 3.  A
// position is one thread's, so the sums do not depend on any order.
template <class Elt, bool kSpans>
__device__ __forceinline__ void add_weights(const PagedArgs& a, const Seen& seen, int n, int b, int h, int v0) {
  const float post = Elt::post_scale(a.scale_log2e);
  const size_t bh = (size_t)b * a.heads + h;
  f32x4 w = {0.f, 0.f, 0.f, 0.f};
  for (int g = 0; g < a.group; ++g) {
    const size_t head = bh * (size_t)a.group + (size_t)g;
    const f32x2 ml = *reinterpret_cast<const f32x2*>(a.final_ml + 2 * head);
    const f32x4 s = *reinterpret_cast<const f32x4*>(a.scores + head * (size_t)a.max_len + (size_t)v0);
    const float inv = ml[1] != 0.f ? 1.f / ml[1] : 0.f;
    const float safe = ml[0] == -INFINITY ? 0.f : ml[0];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = fmaf(__builtin_amdgcn_exp2f((s[k] - safe) * post), inv, w[k]);
  }
  float* row = a.weights + bh * (size_t)a.max_len;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int v = v0 + k;
    if (v < n) {
      const int p = kSpans ? a.list[(size_t)b * a.max_len + v] : (v < seen.sinks ? v : v - seen.sinks + seen.low);
      row[p] += w[k];
    }
  }
}

// kWeights: a call that adds up weights.  (Code that is jumped over is fetched all the same: without weights the few microseconds of the smallest calls
// are 0.3 to 0.7 shorter for its absence.)
template <class Elt, int D, PagedKind kKind, bool kWeights, class Args>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(PagedShape<Elt, D>::kWaves, PagedShape<Elt, D>::kWaves))) void paged_kernel(const Args a) {
  using Shape = PagedShape<Elt, D>;
  constexpr bool kSpans = kKind == kPagedSpans, kSelected = kKind == kPagedSelected;
  constexpr int NK = Shape::NK, NE = Shape::NE, VW = Shape::VW, S = Shape::S;
  constexpr int TR = 16 * S;  // rows of a step
  constexpr uint32_t ROWB = Shape::kRowBytes;
  constexpr int kPieces = ROWB / 16;
  constexpr int kQRow = ROWB + 16;  // LDS rows of q, padded: operand reads spread over the banks
  constexpr int kAccRow = D + 4;
  constexpr int kTerms = 3;         // a 16-bit weight as three terms: all 24 bits of the fp32 one
  constexpr int kKSets = NK == 2 ? 1 : 2;  // K loads of eight rows x 128 bytes, see matrix_kernel's load_k
  constexpr bool kSplitPieces = VW == 8;
  static_assert(kPWin % TR == 0, "tiles do not straddle a window");

  priority(0, 0);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qi = lane & 15, c4 = lane >> 4;
  const int h = blockIdx.x, kv_heads = a.heads, group = a.group;

  struct StreamTables {
    int row[kWavesPerBlock][kPWin];  // pool rows (span form: first the positions)
    IntervalTables tab;
    unsigned char q[16 * kQRow] __attribute__((aligned(16)));
  };
  struct WaveStates {
    float acc[kWavesPerBlock][16][kAccRow];
  };
  union Overlaid {
    StreamTables st;
    WaveStates ws;
  };
  __shared__ __attribute__((aligned(16))) Overlaid s_u;
  __shared__ __attribute__((aligned(16))) f32x2 s_ml[16][kWavesPerBlock];
  __shared__ uint32_t s_ticket;
  auto& s_row = s_u.st.row;
  auto& s_q = s_u.st.q;

  Slice sl;
  if constexpr (Args::kHasTable) {
    const uint32_t entry = a.table[blockIdx.y];
    sl = Slice{(int)(entry & 1023u), (int)(entry >> 10 & 2047u), (int)(entry >> 21), 0, 0};
    sl.y0 = (int)blockIdx.y - sl.split;
  } else if (!kSpans && a.room > 0) {
    sl = locate_slice(a, (int)blockIdx.y, lane, [&](int len) {
      return kSelected ? selected_positions(a, len) : seen_by_last(len, a.max_len, a.window, a.sinks).count;
    });
    if (sl.b < 0) return;  // (the grid holds the most slices that any lengths give)
  } else {
    sl.nsl = a.num_splits;
    sl.b = (int)blockIdx.y / sl.nsl;
    sl.split = (int)blockIdx.y - sl.b * sl.nsl;
    sl.y0 = sl.b * sl.nsl;
  }
  const int b = sl.b, split = sl.split, nsl = sl.nsl;
  const size_t bh = (size_t)b * kv_heads + h;
  const int32_t* table = a.block_table + (size_t)b * a.table_pages;

  // Query head j of the group is row (b, h * group + j) of q and out; columns past the group are computed from its last head
  // and never written.
  auto qrow = [&](int j) { return bh * (size_t)group + (size_t)min(j, group - 1); };
  constexpr int kQLoads = (16 * kPieces + kThreads - 1) / kThreads;
  u32x4 q_piece[kQLoads];
#pragma unroll
  for (int i = 0; i < kQLoads; ++i) {
    const int idx = min(tid + i * kThreads, 16 * kPieces - 1);
    q_piece[i] = *reinterpret_cast<const u32x4*>((const char*)a.q + qrow(idx / kPieces) * ROWB + 16u * (uint32_t)(idx % kPieces));
  }
  const float post = Elt::post_scale(a.scale_log2e);  // see matrix_kernel: weight = exp2((score - largest score) * post)

  Intervals intervals = {0, 0, 0, 0, 0};
  Seen seen = {0, 0, 0};
  int n_total;
  if constexpr (kSpans) {
    SequenceWords words;
    words.first = __builtin_amdgcn_readfirstlane(a.offsets[b]);
    words.last = __builtin_amdgcn_readfirstlane(a.offsets[b + 1]);
    intervals = interval_range(a, words);
    fetch_first(a, intervals, lane);
    n_total = clampi(count_positions(a, intervals, wave, lane, s_u.st.tab), 0, a.max_len);
  } else {
    if (a.room == 0) sl.len = __builtin_amdgcn_readfirstlane(a.ctx_lens[b]);
    if constexpr (kSelected) {
      n_total = selected_positions(a, sl.len);
    } else {
      seen = seen_by_last(sl.len, a.max_len, a.window, a.sinks);
      n_total = seen.count;
    }
  }
  n_total = __builtin_amdgcn_readfirstlane(n_total);
  // even shares of whole steps
  const int T = (int)(((uint32_t)(n_total + nsl - 1) / (uint32_t)nsl + kPagedSliceStep - 1) / kPagedSliceStep * kPagedSliceStep);
  const int slice_begin = min((int)min((int64_t)split * T, (int64_t)n_total), n_total);
  const int cnt = __builtin_amdgcn_readfirstlane(min(n_total - slice_begin, T));
  if (kSpans && kWeights && split == 0 && h == 0 && tid == 0) a.counts[b] = n_total;

  // Units of 16 rows are dealt to the waves round-robin (wave w has the slice's units w, w + 4, ...), which take S of them at a step.
  constexpr int kUnit = 16;
  const int units_all = (cnt + kUnit - 1) / kUnit;
  const int units = units_all > wave ? (units_all - wave + kWavesPerBlock - 1) / kWavesPerBlock : 0;
  const bool own_last = units > 0 && wave + (units - 1) * kWavesPerBlock == units_all - 1;
  const int nrows = units * kUnit - (own_last ? units_all * kUnit - cnt : 0);
  const int vbase = slice_begin + wave * kUnit;
  constexpr int kGap = (kWavesPerBlock - 1) * kUnit;
  auto vrow = [&](int r) { return vbase + r + (r / kUnit) * kGap; };

  // Pool rows of the wave's rows w0 .. w0 + wn - 1, and -1 up to the end of their last step.
  auto tabulate = [&](int w0, int wn, int ln) {
    if constexpr (kSpans) {
      if (w0 == 0 && intervals.count <= 64) tabulate_short<kUnit, kPWin>(a, intervals, vbase, kGap, wn, wave, ln, s_u.st.tab, s_row[wave]);
      else tabulate_positions(a, intervals, vrow, w0, wn, wave, ln, s_u.st.tab, s_row[wave]);
    }
    const int padded = (wn + TR - 1) / TR * TR;
    for (int r = ln; r < padded; r += 64) {
      int x = -1;
      if (r < wn) {
        const int v = vrow(w0 + r);
        int p;
        if constexpr (kSpans) p = clampi(s_row[wave][r], 0, a.max_len - 1);  // (a list whose positions add up past 32 bits leaves rows that the walk does not find)
        else if constexpr (kSelected) p = selected_position(a, bh, sl.len, v);
        else p = v < seen.sinks ? v : v - seen.sinks + seen.low;
        if (!kSelected || p >= 0) x = pool_row(table, p, a.page_shift, a.num_pages);
        // (who adds up weights reads his own entries back; the heads' are equal)
        if (kSpans && kWeights && (h == 0 || a.weights_here)) a.list[(size_t)b * a.max_len + v] = p;
      }
      s_row[wave][r] = x;
    }
    wave_lds_order();
  };
  if (nrows > 0) tabulate(0, min(kPWin, nrows), lane);

  const uint32_t in_page = (1u << a.page_shift) - 1u;
  const uint32_t page_skip = (uint32_t)(kv_heads - 1) * ROWB;  // what a page of all heads has more than one of this head, per row
  const size_t head_off = ((size_t)h << a.page_shift) * ROWB;
  const char* k_head = (const char*)a.k + head_off;
  const char* v_head = (const char*)a.v + head_off;
  auto row_offset = [&](int x) -> uint64_t {  // rows that take no part: the pool's first, whose values are not used
    const uint32_t u = x < 0 ? 0u : (uint32_t)x;
    return (uint64_t)u * ROWB + (uint64_t)(u & ~in_page) * page_skip;
  };

  float ref = -INFINITY, lsum = 0.f;
  f32x4 O[NE];
#pragma unroll
  for (int e = 0; e < NE; ++e) O[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto column = [&](int i, int u) { return kSplitPieces ? 64 * u + 4 * i : NE * i + 4 * u; };

  u32x4 kr[S][NK];
  uint32_t vr[S][4][VW];
  struct TileRows {   // wave-uniform
    uint32_t ok[S];   // bit i: row 16 s + i takes part
    bool plain;       // all of them do
  };
  auto load_k = [&](int base, int ln) {
    const int qi = ln & 15, c4 = ln >> 4;
    TileRows tr;
    tr.plain = true;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      constexpr int kRows = 16 / kKSets;
      global_u32x4 at[kKSets];
      tr.ok[s] = 0;
#pragma unroll
      for (int i = 0; i < kKSets; ++i) {
        const int x = s_row[wave][base + 16 * s + kRows * i + qi % kRows];
        tr.ok[s] |= ((uint32_t)__builtin_amdgcn_ballot_w64(x >= 0) & ((1u << kRows) - 1u)) << (kRows * i);
        at[i] = (global_u32x4)(uintptr_t)(k_head + row_offset(x) + 64u * (uint32_t)(qi / kRows) + 16u * (uint32_t)c4);
      }
      tr.plain = tr.plain && tr.ok[s] == 0xffffu;
#pragma unroll
      for (int mm = 0; mm < NK; ++mm) kr[s][mm] = __builtin_nontemporal_load(at[mm % kKSets] + 4 * kKSets * (mm / kKSets));
    }
    return tr;
  };
  auto order_k = [&]() {  // (as in matrix_kernel: lanes i and i + 8 swap line halves)
    if constexpr (kKSets == 2) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int j = 0; j < NK / 2; ++j) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t x = kr[s][2 * j][k], y = kr[s][2 * j + 1][k];
            kr[s][2 * j][k] = swap_half<0xc>(x, y);
            kr[s][2 * j + 1][k] = swap_half<0x3>(y, x);
          }
        }
      }
    }
  };
  auto load_v = [&](int base, int ln) {
    const int qi = ln & 15, c4 = ln >> 4;
    const uint32_t in_row = (kSplitPieces ? 16u : (uint32_t)(VW * 4)) * (uint32_t)qi;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const i32x4 x4 = *reinterpret_cast<const i32x4*>(&s_row[wave][base + 16 * s + 4 * c4]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const char* at = v_head + row_offset(x4[t]) + in_row;
        if constexpr (VW == 2) {
          const u32x2 w = __builtin_nontemporal_load((global_u32x2)(uintptr_t)at);
          vr[s][t][0] = w[0];
          vr[s][t][1] = w[1];
        } else {
#pragma unroll
          for (int u = 0; u < VW / 4; ++u) {
            const u32x4 w = __builtin_nontemporal_load((global_u32x4)(uintptr_t)(at + 256 * u));
#pragma unroll
            for (int k = 0; k < 4; ++k) vr[s][t][4 * u + k] = w[k];
          }
        }
      }
    }
  };
  // Unscaled scores of the tile in kr: sc[s][t] = column qi against row 16 s + 4 c4 + t.
  auto take_scores = [&](f32x4 (&sc)[S]) {
    constexpr f32x4 kZero = {0.f, 0.f, 0.f, 0.f};
    order_k();
    const unsigned char* qrow_lds = &s_q[qi * kQRow + 16 * c4];
    if constexpr (Elt::kBytes == 2) {
#pragma unroll
      for (int s = 0; s < S; ++s) sc[s] = kZero;
#pragma unroll
      for (int mm = 0; mm < NK; ++mm) {
        const u32x4 qm = *reinterpret_cast<const u32x4*>(qrow_lds + 64 * mm);
#pragma unroll
        for (int s = 0; s < S; ++s) sc[s] += Elt::mfma(kr[s][mm], qm, kZero);
      }
    } else {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        f32x4 sum[4] = {kZero, kZero, kZero, kZero};
#pragma unroll
        for (int mm = 0; mm < NK; ++mm) {
          const u32x4 qm = *reinterpret_cast<const u32x4*>(qrow_lds + 64 * mm);
          f32x4 piece[2] = {kZero, kZero};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t kw = kr[s][mm][k], qw = qm[k];
            piece[k & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, kw), __builtin_bit_cast(float, qw), piece[k & 1], 0, 0, 0);
          }
          sum[mm & 3] += piece[0] + piece[1];
        }
        sc[s] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        pin(sc[s]);
      }
    }
  };
  const __amdgpu_buffer_rsrc_t pair_scores = slab_resource(a.scores + bh * (size_t)group * (size_t)a.max_len, kWeights ? (uint32_t)group * (uint32_t)a.max_len * 4u : 0u);
  // Scores -> weights; moves the state's maximum and adds to its sum.  v0: virtual position of the step's first row.
  auto softmax_step = [&](f32x4 (&sc)[S], int v0, const TileRows& tr) {
    if (!tr.plain) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[s][t] = (tr.ok[s] >> (4 * c4 + t)) & 1u ? sc[s][t] : -INFINITY;
      }
    }
    if constexpr (kWeights) {
      // (Stores without a branch: the waits for the rows behind them are counted.  What is nobody's, or the next slice's, goes out of the descriptor's range.)
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const int v = v0 + kWavesPerBlock * kUnit * s + 4 * c4;  // (s > 0: the wave's next unit)
        const uint32_t at = qi < group && v < slice_begin + cnt ? ((uint32_t)qi * (uint32_t)a.max_len + (uint32_t)v) * 4u : ~15u;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sc[s]), pair_scores, at, 0, 0);
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int t = 0; t < 4; ++t) mx = fmaxf(mx, sc[s][t]);
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
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[s][t] = __builtin_amdgcn_exp2f((sc[s][t] - ref_safe) * post);
      lsum += (sc[s][0] + sc[s][1]) + (sc[s][2] + sc[s][3]);
    }
  };
  auto add_outputs = [&](const f32x4 (&w)[S], const TileRows& tr) {
    if (!tr.plain) {  // what was loaded for rows that take no part must not meet a weight of zero
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int k = 0; k < VW; ++k) vr[s][t][k] = (tr.ok[s] >> (4 * c4 + t)) & 1u ? vr[s][t][k] : 0u;
        }
      }
    }
    if constexpr (Elt::kBytes == 2) {
      uint32_t terms[kTerms][2 * S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t tt[kTerms];
          Elt::template split<kTerms>(w[s][2 * k] * Elt::kWeightScale, w[s][2 * k + 1] * Elt::kWeightScale, tt);
#pragma unroll
          for (int i = 0; i < kTerms; ++i) terms[i][2 * s + k] = tt[i];
        }
      }
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
        uint32_t va[2 * S];
#pragma unroll
        for (int s = 0; s < S; ++s) {
          va[2 * s] = __builtin_amdgcn_perm(vr[s][1][e >> 1], vr[s][0][e >> 1], sel);
          va[2 * s + 1] = __builtin_amdgcn_perm(vr[s][3][e >> 1], vr[s][2][e >> 1], sel);
        }
        f32x4 part = D == 64 ? f32x4{0.f, 0.f, 0.f, 0.f} : O[e];
#pragma unroll
        for (int i = kTerms - 1; i >= 0; --i) {
          if constexpr (S == 1) part = Elt::mfma(u32x2{va[0], va[1]}, u32x2{terms[i][0], terms[i][1]}, part);
#pragma unroll
          for (int s = 0; s + 1 < S; s += 2)
            part = Elt::mfma(u32x4{va[2 * s], va[2 * s + 1], va[2 * s + 2], va[2 * s + 3]},
                             u32x4{terms[i][2 * s], terms[i][2 * s + 1], terms[i][2 * s + 2], terms[i][2 * s + 3]}, part);
        }
        O[e] = D == 64 ? O[e] + part : part;
        if (D == 64) pin(O[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        f32x4 part[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < S; ++s) {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t vw = vr[s][t][e];
            part[t & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, vw), w[s][t], part[t & 1], 0, 0, 0);
          }
        }
        O[e] += part[0] + part[1];
        pin(O[e]);
      }
    }
  };

  TileRows cur = {};
  if (nrows > 0) {
    cur = load_k(0, lane);
    load_v(0, lane);
  }
#pragma unroll
  for (int i = 0; i < kQLoads; ++i) {
    const int idx = tid + i * kThreads, j = idx / kPieces;
    if (16 * kPieces % kThreads != 0 && idx >= 16 * kPieces) continue;
    for (int k = 0; k < 4; ++k) q_piece[i][k] = Elt::scale_query(q_piece[i][k], a.scale_log2e);
    *reinterpret_cast<u32x4*>(&s_q[j * kQRow + 16u * (uint32_t)(idx % kPieces)]) = q_piece[i];
  }
  __syncthreads();  // q is in LDS
  const int quarter = max((nrows / 4 + TR - 1) / TR * TR, TR);
  for (int w0 = 0; w0 < nrows; w0 += kPWin) {
    const int wn = min(kPWin, nrows - w0);
    if (__builtin_expect(w0 > 0, 0)) {
      int ln = lane;
      asm volatile("" : "+v"(ln));  // (the addresses are computed here and not kept across the tiles)
      tabulate(w0, wn, ln);
      cur = load_k(0, ln);
      load_v(0, ln);
    }
    int base = 0;
    for (; base + TR < wn; base += TR) {
      f32x4 sc[S];
      if (w0 + base > 0) priority(w0 + base, quarter);
      take_scores(sc);
      const TileRows next = load_k(base + TR, lane);
      softmax_step(sc, vrow(w0 + base), cur);
      add_outputs(sc, cur);
      load_v(base + TR, lane);
      cur = next;
      asm volatile("" ::"v"(lsum) : "memory");  // (the next tile's work stays behind)
    }
    f32x4 sc[S];
    take_scores(sc);
    softmax_step(sc, vrow(w0 + base), cur);
    add_outputs(sc, cur);
  }

  // ---- the waves' states, and the slices', are merged --------------------------------------------------
  lsum = across_groups_sum<16>(lsum) * Elt::kWeightScale;
  if (c4 == 0) s_ml[qi][wave] = f32x2{ref, lsum};
  const bool whole = finish_pair<D, kWeights, 1>(a, sl, h, post, Elt::kWeightScale, s_ml, s_u.ws.acc, s_ticket, [&](float (&acc)[16][kAccRow]) {
    if (qi < group) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int u = 0; u < NE / 4; ++u)
          *reinterpret_cast<f32x4*>(&acc[qi][column(4 * c4 + r, u)]) = f32x4{O[4 * u][r], O[4 * u + 1][r], O[4 * u + 2][r], O[4 * u + 3][r]};
      }
    }
  });
  if (kWeights && whole && a.weights_here) {  // (no sequence of the call is cut: nothing else is waited for)
    __syncthreads();                          // scores, list and final states are written
    for (int v0 = 4 * tid; v0 < n_total; v0 += 4 * kThreads) add_weights<Elt, kSpans>(a, seen, n_total, b, h, v0);
  }
}

template <class Elt, bool kSpans>
__global__ __launch_bounds__(256) void weights_kernel(const PagedArgs a) {
  const int h = blockIdx.y, b = blockIdx.z;
  const int v0 = 4 * (int)(blockIdx.x * 256 + threadIdx.x);
  Seen seen = {0, 0, 0};
  int n;
  if constexpr (kSpans) n = a.counts[b];
  else {
    seen = seen_by_last(a.ctx_lens[b], a.max_len, a.window, a.sinks);
    n = seen.count;
  }
  if (v0 < n) add_weights<Elt, kSpans>(a, seen, n, b, h, v0);
}

__global__ __launch_bounds__(256) void clear_words_kernel(uint32_t* p, size_t n) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0u;
}


template <class Elt, int D, PagedKind kKind>
int run_paged(const PagedArgs& base, const PagedPlan& p, const uint32_t* table, hipStream_t stream) {
  const dim3 grid((unsigned)base.heads, (unsigned)p.rows);
  auto start = [&](const auto& a) {
    using Args = std::decay_t<decltype(a)>;
    if constexpr (kKind != kPagedSelected) {
      if (a.weights != nullptr) {
        hipLaunchKernelGGL((paged_kernel<Elt, D, kKind, true, Args>), grid, dim3(kThreads), 0, stream, a);
        return;
      }
    }
    hipLaunchKernelGGL((paged_kernel<Elt, D, kKind, false, Args>), grid, dim3(kThreads), 0, stream, a);
  };
  PagedArgsPlain plain;
  static_cast<PagedArgs&>(plain) = base;
  if constexpr (kKind == kPagedSpans) {  // (the others find their slices on the device)
    if (p.table) {
      PagedArgsTable a;
      static_cast<PagedArgs&>(a) = base;
      for (int32_t i = 0; i < p.rows; ++i) a.table[i] = table[i];
      start(a);
    } else {
      start(plain);
    }
  } else {
    start(plain);
  }
  const int rc = launched();
  if (rc != SPAN_OK || base.weights == nullptr || base.weights_here) return rc;
  int64_t most = base.max_len;
  if (kKind == kPagedDense && base.window > 0 && (int64_t)base.window + base.sinks < most) most = (int64_t)base.window + base.sinks;
  hipLaunchKernelGGL((weights_kernel<Elt, kKind == kPagedSpans>), dim3((unsigned)((most + 1023) / 1024), (unsigned)base.heads, (unsigned)base.batch), dim3(256), 0,
                     stream, base);
  return launched();
}

template <PagedKind kKind>
int paged_decode(const span_paged_desc_t* d, const void* q, const void* k, const void* v, const int32_t* block_table, const int32_t* ctx_lens,
                 const int32_t* offsets, const int32_t* starts, const int32_t* ends, const int32_t* selected, float scale, float* weights, float* out) {
  PagedArgs a;
  PagedPlan p;
  uint32_t table[kMaxPlanSlices];
  const int rc = one_token_args(d, kKind, q, k, v, block_table, ctx_lens, offsets, starts, ends, selected, scale, weights, out, &a, &p, table);
  if (rc != SPAN_OK) return rc;
  hipStream_t stream = (hipStream_t)d->stream;
  const bool d128 = d->head_dim == 128;
  switch (d->dtype) {
    case SPAN_F32:
      return d128 ? run_paged<F32, 128, kKind>(a, p, table, stream) : run_paged<F32, 64, kKind>(a, p, table, stream);
    case SPAN_F16:
      return d128 ? run_paged<F16, 128, kKind>(a, p, table, stream) : run_paged<F16, 64, kKind>(a, p, table, stream);
    default:
      return d128 ? run_paged<BF16, 128, kKind>(a, p, table, stream) : run_paged<BF16, 64, kKind>(a, p, table, stream);
  }
}

}  // namespace
}  // namespace spanattn

extern "C" int paged_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                                 const int32_t* ctx_lens, float scale, float* weights, float* out) {
  return spanattn::paged_decode<spanattn::kPagedDense>(desc, q, k_pages, v_pages, block_table, ctx_lens, nullptr, nullptr, nullptr, nullptr, scale, weights, out);
}

extern "C" int paged_span_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                                      const int32_t* block_table, const int32_t* span_offsets, const int32_t* span_starts,
                                      const int32_t* span_ends, float scale, float* weights, float* out) {
  return spanattn::paged_decode<spanattn::kPagedSpans>(desc, q, k_pages, v_pages, block_table, nullptr, span_offsets, span_starts, span_ends, nullptr, scale,
                                                       weights, out);
}

extern "C" int paged_selected_decode_attn(const span_paged_desc_t* desc, const void* q, const void* k_pages, const void* v_pages,
                                          const int32_t* block_table, const int32_t* ctx_lens, const int32_t* selected, float scale, float* out) {
  return spanattn::paged_decode<spanattn::kPagedSelected>(desc, q, k_pages, v_pages, block_table, ctx_lens, nullptr, nullptr, nullptr, selected, scale,
                                                          nullptr, out);
}

extern "C" int paged_workspace_init(const span_paged_desc_t* desc) {
  const int rc = spanattn::check_paged(desc);
  if (rc != SPAN_OK) return rc;
  const size_t bytes = spanattn::counter_bytes(desc);
  if (!desc->workspace || ((uintptr_t)desc->workspace & 255u) || desc->workspace_bytes < bytes) return SPAN_ERR_WORKSPACE;
  const size_t words = bytes / sizeof(uint32_t);
  hipLaunchKernelGGL(spanattn::clear_words_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, (hipStream_t)desc->stream,
                     (uint32_t*)desc->workspace, words);
  return spanattn::launched();
}
