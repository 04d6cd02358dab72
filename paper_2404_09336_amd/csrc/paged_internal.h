// Shared by the translation units of the operators on a cache in pages.
#ifndef PAGED_INTERNAL_H_
#define PAGED_INTERNAL_H_

#include "span_internal.h"
#include "span_paged.h"

namespace spanattn {

constexpr int kMaxGroup = 16;          // query heads per KV head: columns of one 16x16 MFMA
constexpr int kPagedSliceStep = 32;    // slices are multiples of this many positions (whole tiles, whole quads of scores)
constexpr int kPagedLeastSlice = 128;  // do not cut finer: a tile per wave
// Dense calls find their slices on the device, from the lengths, every workgroup for itself (locate_slice); beyond this batch that
// takes longer than it gains, and there are workgroups enough without slices.
constexpr int kPagedLocateBatch = 512;

// What a one-token call attends: the cache up to a token (window, sinks), a sequence's span, or the pages listed for a (sequence, KV head).
enum PagedKind { kPagedDense, kPagedSpans, kPagedSelected };

// What host and device count alike (constexpr: code of both).
constexpr int within(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Positions that the token at position n - 1 sees: [0, sinks) and from `low` on, of those below n that the table has.
struct Seen {
  int sinks, low, count;
};
constexpr Seen seen_by_last(int n, int max_len, int window, int sinks) {
  const int held = within(n, 0, max_len), low = window > 0 ? within((n > 0 ? n : 0) - window, 0, held) : 0;
  const int first = sinks < low ? sinks : low;
  return Seen{first, low, held - low + first};
}

// A sequence of up to so many positions is not cut: the hand-over costs more than a workgroup's two or four tiles a wave.
inline int32_t paged_whole(const span_paged_desc_t* d, bool fp4 = false) { return fp4 ? 1024 : d->dtype == SPAN_F32 && d->head_dim == 128 ? 128 : 256; }
// Rows of 4 bits are through four times as fast, and a hand-over (some 3.5 us) costs as much as a thousand of them.  us, 256 positions at least and whole up to 256 -> 512 and 1024: 16 x 32
// pairs of ~500 in spans 15.6 -> 14.1; 64 x 8 of 512 .. 4096 and 4 x 8 of 8000 .. 32768 the same.
// Listed pages have a trip more ahead of their rows.  us, 128 -> 256: 4 x 8 pairs of 2048 positions on 32 pages, four query heads each, 13.9 -> 11.9.
inline int32_t paged_least(PagedKind kind, bool fp4) { return fp4 ? 512 : kind == kPagedSelected ? 2 * kPagedLeastSlice : kPagedLeastSlice; }

int check_paged(const span_paged_desc_t* d);

// Counters at the head of every workspace that has some, zero between calls: of every (sequence, KV head), then of every sequence.
inline size_t counter_bytes(const span_paged_desc_t* d) { return ((size_t)d->batch * (d->kv_heads + 1) * sizeof(int32_t) + 255) & ~(size_t)255; }

inline int page_shift(const span_paged_desc_t* d) { return __builtin_ctz((unsigned)d->page_size); }
inline int32_t capacity(const span_paged_desc_t* d) { return d->table_pages * d->page_size; }  // positions of a sequence's table

// How a one-token call is cut.
struct PagedPlan {
  int32_t room;      // > 0: slices per head the kernel aims at over all sequences (locate_slice; `rows` where that is not level)
  int32_t splits;    // room 0: slices of every sequence, or the most of any (table)
  bool table;        // slices from a table of pack_slice entries
  int32_t rows;      // grid.y: slices of all sequences (upper bound)
  bool cut;          // some lengths give some sequence several slices
  bool own_weights;  // the workgroup that attends adds up the weights too
};
// `table` (kMaxPlanSlices entries) may be null to only size the plan.
// (fp4: of a cache held in 4 bits)
PagedPlan plan_paged(const span_paged_desc_t* d, PagedKind kind, uint32_t* table, bool fp4 = false);
inline PagedPlan plan_paged(const span_paged_desc_t* d, bool spans, uint32_t* table) { return plan_paged(d, spans ? kPagedSpans : kPagedDense, table); }

// Parts of the workspace of a one-token call, in bytes from its start.
struct PagedWorkspace {
  size_t ml, acc, final_ml, counts, list, scores, total;  // counters lie at 0
  bool sliced, weights, spans;
};
PagedWorkspace paged_workspace(const span_paged_desc_t* d, const PagedPlan& p, PagedKind kind, bool weights);
inline PagedWorkspace paged_workspace(const span_paged_desc_t* d, const PagedPlan& p, bool spans, bool weights) {
  return paged_workspace(d, p, spans ? kPagedSpans : kPagedDense, weights);
}

// How a prompt call is cut: query rows in tiles, and a tile's positions among several workgroups where there are few tiles.
constexpr int kPromptTileRows = 128;
struct PromptPlan {
  int32_t tokens;   // of a tile: as many as their heads' rows fit
  int32_t splits;
  int64_t tiles;    // the most that any offsets give
  size_t acc;       // bytes of the workspace ahead of the partial outputs
};
PromptPlan plan_prompt(const span_paged_desc_t* d);
size_t prompt_workspace(const span_paged_desc_t* d, const PromptPlan& p);

// Whether new rows can be turned as `r` (null: not turned) says.
int check_rotation(const span_paged_desc_t* d, const paged_rotation_t* r);

// A page of 4-bit values holds its rows' codes, then their exponents.  Both lie in groups of 16 rows, K's codes by blocks of 32 channels and in each by rows, V's by fours of rows, in
// each by sixteenths of the channels and in those by rows, the exponents by blocks and in each by rows: what a lane of the attention kernel takes is contiguous.
constexpr int kFp4Rows = 16, kFp4Block = 32;  // rows of a group, channels that share an exponent
constexpr int kFp4LeastExponent = -126, kFp4MostExponent = 125;

// A one-token call over such pages goes by units, a group's rows: those of the first `sinks` positions, then those from `low` on.  A unit that both touch is two.
struct SeenUnits {
  int sinks, low, held, first;  // positions; units of the sinks
};
constexpr SeenUnits seen_units(int n, int max_len, int window, int sinks) {
  const Seen s = seen_by_last(n, max_len, window, sinks);
  return SeenUnits{s.sinks, s.low, within(n, 0, max_len), (s.sinks + kFp4Rows - 1) / kFp4Rows};
}
constexpr int unit_count(const SeenUnits& s) { return s.first + (s.held > s.low ? (s.held + kFp4Rows - 1) / kFp4Rows - s.low / kFp4Rows : 0); }
// Positions of the most units that any length has: W positions in a row touch (W + 14) / 16 + 1 of them at most, and of a table's units the one where sinks end and the window begins can be there twice.
constexpr int64_t most_unit_positions(int64_t max_len, int64_t window, int64_t sinks) {
  if (window <= 0) return max_len;
  const int64_t units = (sinks + kFp4Rows - 1) / kFp4Rows + (window + kFp4Rows - 2) / kFp4Rows + 1, table = max_len / kFp4Rows + (sinks > 0 ? 1 : 0);
  return (units < table ? units : table) * kFp4Rows;
}

// Slices of a dense call: sequence b has one, or ceil(n_b / T) of at most T positions if it has more than `whole`, T whole steps and `least` at least.  T starts at the positions of all
// sequences over `room` and grows, by the slices too many in proportion and a sixteenth at least, until no more than `room` are left or no sequence is cut.  If that leaves the longest slice
// well above the mean, which is what the whole call waits for then, `rows` is tried.  More than `rows`, the slices that the grid and the workspace hold, it never gives: a bound of them that is
// too low costs time and nothing else.
// (us, 1024 workgroups always -> 512 and 1024 where those are not level: 32 sequences in a window of 1024 29.0 -> 27.0, four of 8000 .. 32768 72.9 -> 68.7;
// 512 always: 64 x 8 pairs of 512 .. 4096 106.4 -> 112.2.  One round each way: with as many slices as came out, 1.25 rounds, those took 110.9.)
// `all`, `longest`: positions of the sequences; slices(T): all their slices of that length.
template <class Slices>
constexpr __attribute__((always_inline)) uint32_t slice_length(uint32_t all, uint32_t longest, uint32_t batch, uint32_t room, uint32_t rows, uint32_t whole, uint32_t least, Slices&& slices) {
  constexpr uint32_t kStep = kPagedSliceStep;
  uint32_t T = longest;
  if (longest <= whole) return T;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    const uint32_t aim = pass == 0 ? room : rows, most = aim < rows ? aim : rows;
    T = longest;
    if (most > batch) {
      const float mean = (float)all / ((float)aim - 0.5f * (float)batch);  // (a sequence has half a slice more than its share on average)
      T = ((uint32_t)mean + kStep - 1u) / kStep * kStep;
      if (T < least) T = least;
      while (T < longest) {
        const uint32_t total = slices(T);
        if (total <= most) break;
        const uint32_t in_proportion = ((uint32_t)((float)T * (float)total / (float)most) + kStep - 1u) / kStep * kStep, sixteenth = (T + T / 16 + kStep - 1u) / kStep * kStep;
        T = in_proportion > sixteenth ? in_proportion : sixteenth;
        if (T > longest) T = longest;
      }
    }
    const float longest_slice = (float)(T < longest ? T : longest);
    if (longest_slice * (float)(aim > batch ? aim : batch) <= 1.4f * (float)all || T <= least) break;
  }
  return T;
}

// A selection's scores, one of each page of a (sequence, KV head), behind the counters.
int check_select(const span_paged_desc_t* d);
size_t select_workspace(const span_paged_desc_t* d);

// An eviction of longer caches keeps lists in the workspace and moves their rows in a second launch.
constexpr int32_t kMostKeysHeld = 32768;
int32_t most_moves(const span_paged_desc_t* d);  // rows of a (sequence, KV head) that an eviction moves at most
size_t evict_workspace(const span_paged_desc_t* d);

}  // namespace spanattn
#endif
