// Randomised check of the plans of one-token calls on a cache in pages: a plan that says no sequence is cut is right for all lengths, and the
// slices of any lengths have their rows in the grid and their states in the workspace.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "paged_internal.h"

#define REQUIRE(c)                                                        \
  do {                                                                    \
    if (!(c)) {                                                           \
      std::printf("%s:%d: %s (case %d)\n", __FILE__, __LINE__, #c, it);   \
      std::abort();                                                       \
    }                                                                     \
  } while (0)

static std::mt19937 rng(20240409);
static int rnd(int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); }

// Slices of a dense call as its workgroups find them (`n`: positions that each sequence attends).
static int64_t slices_found(const std::vector<int64_t>& n, int64_t room, int64_t more_room, int64_t whole) {
  using namespace spanattn;
  const int64_t batch = (int64_t)n.size();
  int64_t all = 0, longest = 1;
  for (int64_t x : n) all += x, longest = std::max(longest, x);
  auto steps = [](int64_t x) { return (x + kPagedSliceStep - 1) / kPagedSliceStep * kPagedSliceStep; };
  auto total = [&](int64_t T) {
    int64_t s = 0;
    for (int64_t x : n) s += x > whole ? (x + T - 1) / T : 1;
    return s;
  };
  int64_t T = longest;
  if (longest > whole) {
    for (int pass = 0; pass < 2; ++pass) {
      const int64_t aim = pass == 0 ? room : more_room;
      T = longest;
      if (aim > batch) {
        T = std::max<int64_t>(steps((int64_t)((float)all / ((float)aim - 0.5f * (float)batch))), kPagedLeastSlice);
        while (T < longest) {
          const int64_t s = total(T);
          if (s <= aim) break;
          T = std::min(std::max(steps((int64_t)((float)T * (float)s / (float)aim)), steps(T + T / 16)), longest);
        }
      }
      if ((float)std::min(T, longest) * (float)std::max(aim, batch) <= 1.4f * (float)all || T <= kPagedLeastSlice) break;
    }
  }
  return total(T);
}

int main() {
  using namespace spanattn;
  int cut_plans = 0, uncut_with_room = 0, cut_lengths = 0;
  for (int it = 0; it < 40000; ++it) {
    span_paged_desc_t d = {};
    const int heads[] = {1, 2, 3, 8, 16, 32, 96, 1024, 3000};
    d.batch = rnd(0, 3) ? rnd(1, 70) : rnd(1, 700);
    d.kv_heads = heads[rnd(0, 8)];
    d.heads = d.kv_heads * rnd(1, 16);
    d.head_dim = rnd(0, 1) ? 128 : 64;
    d.dtype = rnd(0, 2);
    d.page_size = 16 << rnd(0, 4);
    d.num_pages = 1 << 20;
    d.table_pages = rnd(1, rnd(0, 1) ? 40 : 1000);
    d.window = rnd(0, 2) ? 0 : rnd(1, 3000);
    d.sinks = rnd(0, 1) ? 0 : rnd(0, 100);
    d.num_splits = rnd(0, 9) ? 0 : rnd(1, 300);
    REQUIRE(check_paged(&d) == SPAN_OK);
    const PagedPlan p = plan_paged(&d, false, nullptr);
    REQUIRE(p.rows >= d.batch && p.rows <= 65535 && !p.table);
    const PagedWorkspace w = paged_workspace(&d, p, false, false);
    const size_t states = (size_t)p.rows * (size_t)d.heads;
    if (p.cut) {  // a state of every slice, whole; the counters ahead of them
      ++cut_plans;
      REQUIRE(w.sliced && w.ml >= (size_t)d.batch * (d.kv_heads + 1) * 4);
      REQUIRE(w.acc >= w.ml + states * 2 * sizeof(float) && w.total >= w.acc + states * d.head_dim * sizeof(float));
    }
    uncut_with_room += !p.cut && p.room > 0;
    for (int draw = 0; draw < 6; ++draw) {
      std::vector<int64_t> n(d.batch);
      const int kind = rnd(0, 3);
      for (auto& x : n) {
        x = kind == 0 ? capacity(&d) : kind == 1 ? rnd(0, capacity(&d)) : rnd(0, 19) ? rnd(0, 300) : rnd(0, capacity(&d));
        x = std::min<int64_t>(x, capacity(&d));
        if (d.window > 0) x = std::min<int64_t>(x, (int64_t)d.window + d.sinks);
      }
      const int64_t found = p.room > 0 ? slices_found(n, p.room, p.rows, paged_whole(&d)) : (int64_t)p.splits * d.batch;
      REQUIRE(found <= p.rows);
      if (!p.cut) REQUIRE(found == d.batch);
      cut_lengths += found > d.batch;
    }
  }
  std::printf("host_paged_plan: ok, %d cut, %d never for their batch, %d lengths cut\n", cut_plans, uncut_with_room, cut_lengths);
  return cut_plans > 1000 && uncut_with_room > 1000 && cut_lengths > 1000 ? 0 : 1;
}
