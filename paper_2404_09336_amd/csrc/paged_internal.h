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

// A sequence of up to so many positions is not cut: the hand-over costs more than a workgroup's two or four tiles a wave.
inline int32_t paged_whole(const span_paged_desc_t* d) { return d->dtype == SPAN_F32 && d->head_dim == 128 ? 128 : 256; }

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
PagedPlan plan_paged(const span_paged_desc_t* d, bool spans, uint32_t* table);

// Parts of the workspace of a one-token call, in bytes from its start.
struct PagedWorkspace {
  size_t ml, acc, final_ml, counts, list, scores, total;  // counters lie at 0
  bool sliced, weights, spans;
};
PagedWorkspace paged_workspace(const span_paged_desc_t* d, const PagedPlan& p, bool spans, bool weights);

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

// An eviction of longer caches keeps lists in the workspace and moves their rows in a second launch.
constexpr int32_t kMostKeysHeld = 32768;
int32_t most_moves(const span_paged_desc_t* d);  // rows of a (sequence, KV head) that an eviction moves at most
size_t evict_workspace(const span_paged_desc_t* d);

}  // namespace spanattn
#endif
