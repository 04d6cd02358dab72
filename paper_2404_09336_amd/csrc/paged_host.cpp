// Host-only parts of the operators on a cache in pages: argument checks, slices, workspaces.  No GPU call in this file.
#include <limits.h>

#include <algorithm>

#include "paged_internal.h"

namespace spanattn {

int check_paged(const span_paged_desc_t* d) {
  if (!d) return SPAN_ERR_NULL;
  if (d->batch <= 0 || d->batch > 65535 || d->heads <= 0 || d->kv_heads <= 0 || d->kv_heads > 65535) return SPAN_ERR_SHAPE;
  if (d->heads % d->kv_heads != 0 || d->heads / d->kv_heads > kMaxGroup) return SPAN_ERR_SHAPE;
  if (d->head_dim != 64 && d->head_dim != 128) return SPAN_ERR_SHAPE;
  if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0) return SPAN_ERR_SHAPE;
  if (d->num_pages <= 0 || (int64_t)d->num_pages * d->page_size > INT_MAX) return SPAN_ERR_SHAPE;
  if (d->table_pages <= 0 || (int64_t)d->table_pages * d->page_size > kMaxLen) return SPAN_ERR_SHAPE;
  if ((int64_t)d->batch * d->heads > INT_MAX / 2) return SPAN_ERR_SHAPE;
  if (d->num_tokens < 0 || d->window < 0 || d->sinks < 0 || d->num_intervals < 0 || d->num_splits < 0 || d->budget < 0 || d->recent < 0)
    return SPAN_ERR_SHAPE;
  if (d->dtype != SPAN_F32 && d->dtype != SPAN_F16 && d->dtype != SPAN_BF16) return SPAN_ERR_DTYPE;
  return SPAN_OK;
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Workgroups a one-token call aims at: two per CU, and as many as run at once (four) where that leaves slices of very different length.
constexpr int64_t kPagedWorkgroups = 512, kPagedMoreWorkgroups = 1024;

// A dense call that is never cut leaves the weights to a second launch beyond so many positions of all (sequence, KV head) pairs: the launch costs some 3 us, a
// workgroup's own pass over its positions a trip to memory for each 1024.  us, second launch -> own: 128 x 8 pairs in a window of 512 (0.5 M positions at most) 54.8 ->
// 51.6; 64 x 32 of up to 512 (1.0 M) 61.9 -> 60.9; of up to 1472 (3.0 M) 100.5 -> 102.0; of up to 2048 134.8 -> 138.3; 40 x 32 of up to 2000 (2.6 M), four query
// heads each, 115.5 -> 110.7.
constexpr int64_t kPagedOwnWeights = 3 << 19;

PagedPlan plan_paged(const span_paged_desc_t* d, bool spans, uint32_t* table) {
  PagedPlan p = {0, 1, false, 0, false, false};
  const int64_t cap = capacity(d), whole = paged_whole(d);
  const int64_t room = std::max<int64_t>(1, kPagedWorkgroups / d->kv_heads), more_room = std::max<int64_t>(1, kPagedMoreWorkgroups / d->kv_heads);
  auto uniform = [&](int64_t splits) {
    splits = std::min(splits, ceil_div(cap, kPagedSliceStep));
    splits = std::min<int64_t>(splits, 65535 / d->batch);  // grid.y
    p.splits = (int32_t)std::max<int64_t>(splits, 1);
    p.rows = p.splits * d->batch;
    p.cut = p.splits > 1;
    p.own_weights = !p.cut;
    return p;
  };
  if (d->num_splits > 0) return uniform(d->num_splits);
  if (!spans) {
    if (d->batch > kPagedLocateBatch) return uniform(1);
    const int64_t most = d->window > 0 ? std::min<int64_t>(cap, (int64_t)d->window + d->sinks) : cap;  // positions of any sequence
    if (most <= whole) return uniform(1);
    p.room = (int32_t)room;
    p.splits = 2;
    p.rows = (int32_t)std::max<int64_t>(d->batch, std::min<int64_t>(more_room, ceil_div(most, kPagedLeastSlice) * d->batch));
    p.cut = more_room > d->batch;  // (otherwise one slice each whatever the lengths; the workspace is that of other batches of the shape)
    p.own_weights = !p.cut && most * d->batch * d->kv_heads <= kPagedOwnWeights;
    return p;
  }
  if (d->tokens_per_seq && d->batch <= kMaxPlanSlices) {  // as locate_slice does
    auto tokens = [&](int32_t b) { return std::min(std::max<int64_t>(d->tokens_per_seq[b], 0), cap); };
    int64_t sum = 0, longest = 1;
    for (int32_t b = 0; b < d->batch; ++b) {
      sum += tokens(b);
      longest = std::max(longest, tokens(b));
    }
    int64_t T = longest;
    auto slices = [&](int32_t b) { return tokens(b) > whole ? ceil_div(tokens(b), T) : 1; };
    for (const int64_t aim : {room, more_room}) {
      const int64_t most = std::min<int64_t>(aim, kMaxPlanSlices);
      T = longest;
      if (most > d->batch) {
        T = std::max<int64_t>(kPagedLeastSlice, round_up(2 * sum / (2 * most - d->batch), kPagedSliceStep));
        while (T < longest) {
          int64_t total = 0;
          for (int32_t b = 0; b < d->batch; ++b) total += slices(b);
          if (total <= most) break;
          T = std::min(std::max(round_up(T * total / most, kPagedSliceStep), round_up(T + T / 16, kPagedSliceStep)), longest);
        }
      }
      if (std::min(T, longest) * std::max<int64_t>(most, d->batch) * 5 <= 7 * sum || T <= kPagedLeastSlice) break;
    }
    int64_t most = 1, least = kMaxPlanSplits, y = 0;
    for (int32_t b = 0; b < d->batch; ++b) {
      const int64_t nsl = slices(b);
      most = std::max(most, nsl);
      least = std::min(least, nsl);
      y += nsl;
    }
    if (most == least) return uniform(most);
    if (y <= kMaxPlanSlices && most <= kMaxPlanSplits) {
      if (table) {
        int32_t at = 0;
        for (int32_t b = 0; b < d->batch; ++b) {
          const int64_t nsl = slices(b);
          for (int64_t s = 0; s < nsl; ++s) table[at++] = pack_slice((uint32_t)b, (uint32_t)s, (uint32_t)nsl);
        }
      }
      p.table = p.cut = true;
      p.splits = (int32_t)most;
      p.rows = (int32_t)y;
      return p;
    }
  }
  return uniform(std::min(ceil_div(room, d->batch), ceil_div(cap, kPagedLeastSlice)));
}

PagedWorkspace paged_workspace(const span_paged_desc_t* d, const PagedPlan& p, bool spans, bool weights) {
  PagedWorkspace w = {};
  w.sliced = p.splits > 1;
  w.weights = weights;
  w.spans = spans;
  const size_t group = (size_t)(d->heads / d->kv_heads), states = (size_t)p.rows * d->kv_heads * group, cap = (size_t)capacity(d);
  size_t at = 0;
  auto part = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  if (w.sliced || weights) part(counter_bytes(d));
  w.ml = part(w.sliced ? states * 2 * sizeof(float) : 0);
  w.acc = part(w.sliced ? states * (size_t)d->head_dim * sizeof(float) : 0);
  w.final_ml = part(weights ? (size_t)d->batch * d->heads * 2 * sizeof(float) : 0);
  w.counts = part(weights && spans ? (size_t)d->batch * sizeof(int32_t) : 0);
  w.list = part(weights && spans ? (size_t)d->batch * cap * sizeof(int32_t) : 0);
  w.scores = part(weights ? (size_t)d->batch * d->heads * cap * sizeof(float) : 0);
  w.total = at;
  return w;
}

// A prompt call of fewer workgroups than CUs has its tiles' positions shared out, among as many workgroups as kPromptWorkgroups16 / 32 allow and so that each has
// about kPromptLeastPositions16 / 32 of a full table at least; a second launch joins the shares.  fp32 products take eight times as long, so that a share of two steps pays and one workgroup
// keeps a CU busy.  us, bf16 / fp32:
//   never shared                 200 new of 4000, 32 heads on 8 of 128   99 /  -     64 of 3000, 8 heads of 128, fp32     - / 416
//   256 workgroups                                                       39 /  -                                          - /  29 (64 positions at least)
//   512 workgroups                                                       36 /  -                                          - /  35
//   1024 workgroups                                                      48 /  -
//   128, 192, 256 at least (512) 100 of 1000, 8 heads of 128      13, 14, 16 /  -     10 of 6000, 5 heads of 64    15, 14, 14 /  -
//   64, 256 at least (fp32)      100 of 1000, 8 heads of 128           - / 22, 46
constexpr int64_t kPromptFewTiles = 256;
constexpr int64_t kPromptWorkgroups16 = 512, kPromptLeastPositions16 = 192;
constexpr int64_t kPromptWorkgroups32 = 256, kPromptLeastPositions32 = 64;

PromptPlan plan_prompt(const span_paged_desc_t* d) {
  PromptPlan p;
  const int32_t group = d->heads / d->kv_heads;
  p.tokens = kPromptTileRows / group;
  // each sequence has at most one tile that is not full
  p.tiles = (int64_t)d->num_tokens / p.tokens + std::min(d->batch, d->num_tokens);
  const int64_t workgroups = p.tiles * d->kv_heads;
  int64_t most = capacity(d);
  if (d->window > 0) most = std::min<int64_t>(most, (int64_t)d->window + d->sinks + p.tokens);
  int64_t splits = 1;
  const bool fp32 = d->dtype == SPAN_F32;
  if (workgroups > 0 && workgroups < kPromptFewTiles) {
    const int64_t least = fp32 ? kPromptLeastPositions32 : kPromptLeastPositions16;
    splits = std::min((fp32 ? kPromptWorkgroups32 : kPromptWorkgroups16) / workgroups, (most + least / 2) / least);
  }
  p.splits = (int32_t)std::max<int64_t>(splits, 1);
  const size_t rows = p.splits > 1 ? (size_t)workgroups * p.splits * kPromptTileRows : 0;
  p.acc = (rows * 2 * sizeof(float) + 255) & ~(size_t)255;
  return p;
}

size_t prompt_workspace(const span_paged_desc_t* d, const PromptPlan& p) {
  if (p.splits == 1) return 0;
  return p.acc + (size_t)p.tiles * d->kv_heads * p.splits * kPromptTileRows * d->head_dim * sizeof(float);
}

int32_t most_moves(const span_paged_desc_t* d) { return std::min(d->budget, std::max(capacity(d) - d->budget, 0)); }

// The counters, and for long caches of every (sequence, KV head) the number of rows that move and the pairs of their slots (8 bytes each).
size_t evict_workspace(const span_paged_desc_t* d) {
  const size_t lists = capacity(d) > kMostKeysHeld ? (size_t)d->batch * d->kv_heads * (2 + 2 * (size_t)most_moves(d)) * sizeof(int32_t) : 0;
  return (counter_bytes(d) + lists + 255) & ~(size_t)255;
}

}  // namespace spanattn

extern "C" int paged_check(const span_paged_desc_t* desc) { return spanattn::check_paged(desc); }

extern "C" size_t paged_workspace_bytes(const span_paged_desc_t* desc, int use) {
  using namespace spanattn;
  if (check_paged(desc) != SPAN_OK) return 0;
  if (use == PAGED_EVICT) return evict_workspace(desc);
  if (use == PAGED_PROMPT) return prompt_workspace(desc, plan_prompt(desc));
  if (use < PAGED_DECODE || use > PAGED_SPAN_DECODE_WEIGHTS) return 0;
  const bool spans = use >= PAGED_SPAN_DECODE;
  return paged_workspace(desc, plan_paged(desc, spans, nullptr), spans, (use & 1) != 0).total;
}
