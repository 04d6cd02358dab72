// The slices of windowed one-token calls over 4-bit pages against the plan, for windows and sinks around every multiple of a slice's least length and every remainder of a length by a unit's
// rows: each has its row in the grid and its state in the workspace, and the plan's bound alone sees to that.  And the rule itself: it gives no more slices than the grid has, however low its bound.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "paged_internal.h"

using namespace spanattn;

static const char* at = "";
static span_paged_desc_t d;
#define REQUIRE(c)                                                                                                                                          \
  do {                                                                                                                                                      \
    if (!(c)) {                                                                                                                                             \
      std::printf("%s:%d: %s (%s; batch %d, kv heads %d, table %d, window %d, sinks %d)\n", __FILE__, __LINE__, #c, at, d.batch, d.kv_heads, capacity(&d), d.window, d.sinks); \
      std::fflush(stdout);                                                                                                                                  \
      std::abort();                                                                                                                                         \
    }                                                                                                                                                       \
  } while (0)

// Slices of sequences that attend so many positions, as the workgroups of a call find them.
static int64_t slices_found(const std::vector<int64_t>& n, uint32_t room, uint32_t rows, uint32_t whole, uint32_t least) {
  uint32_t all = 0, longest = 1;
  for (int64_t x : n) all += (uint32_t)x, longest = std::max(longest, (uint32_t)x);
  auto total = [&](uint32_t T) {
    uint32_t s = 0;
    for (int64_t x : n) s += x > whole ? ((uint32_t)x + T - 1) / T : 1;
    return s;
  };
  return total(slice_length(all, longest, (uint32_t)n.size(), room, rows, whole, least, total));
}

static int64_t counted(int len) { return (int64_t)unit_count(seen_units(len, capacity(&d), d.window, d.sinks)) * kFp4Rows; }

int main() {
  std::mt19937 rng(20240409);
  auto rnd = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  const int64_t whole = paged_whole(&d, true), least = paged_least(kPagedDense, true);
  int64_t calls = 0, cut = 0, bounded = 0;
  auto check = [&](const std::vector<int>& lens) {
    REQUIRE(check_paged(&d) == SPAN_OK);
    const PagedPlan p = plan_paged(&d, kPagedDense, nullptr, true);
    const PagedWorkspace w = paged_workspace(&d, p, kPagedDense, false);
    const size_t states = (size_t)p.rows * (size_t)d.heads;
    REQUIRE(p.rows >= d.batch && p.rows <= 65535);
    if (p.cut) REQUIRE(w.acc >= w.ml + states * 2 * sizeof(float) && w.total >= w.acc + states * d.head_dim * sizeof(float));
    std::vector<int64_t> n;
    for (int len : lens) {
      n.push_back(counted(len));
      REQUIRE(n.back() <= most_unit_positions(capacity(&d), d.window, d.sinks));
      // Where the plan has all the rows that the least slices need, a sequence's need no more than its share.
      if (p.cut && p.rows < std::max(1, 1024 / d.kv_heads) && p.rows > d.batch) {
        ++bounded;
        REQUIRE((n.back() + least - 1) / least <= p.rows / d.batch);
      }
    }
    if (!p.cut || p.room == 0) return;
    const int64_t found = slices_found(n, (uint32_t)p.room, (uint32_t)p.rows, (uint32_t)whole, (uint32_t)least);
    REQUIRE(found <= p.rows);
    ++calls;
    cut += found > d.batch;
  };
  d.head_dim = 128;
  d.dtype = SPAN_BF16;
  d.num_pages = 1 << 20;
  d.page_size = 16;

  at = "grid";
  for (const int kv : {1, 2, 8, 32}) {
    for (const int batch : {1, 4, 7, 16, 32, 65}) {
      d.batch = batch;
      d.kv_heads = kv;
      d.heads = 4 * kv;
      for (int step = 2; step <= 9; ++step) {
        for (const int off : {-33, -32, -31, -17, -16, -15, -6, -4, -1, 0, 1, 2, 15, 16, 17}) {
          for (const int sinks : {0, 1, 4, 15, 16, 17, 31, 64}) {
            for (const bool together : {false, true}) {  // the window alone, or window and sinks, near the multiple
              d.sinks = sinks;
              d.window = 512 * step + off - (together ? sinks : 0);
              for (const int table : {d.window / 16 + 1, (d.window + sinks) / 16 + 1, (d.window + sinks) / 16 + 2, 2000}) {
                d.table_pages = table;
                for (int r = 0; r < 16; ++r) check(std::vector<int>(batch, std::min(d.window + sinks + 1000, 16 * table - 16) / 16 * 16 + r));
              }
            }
          }
        }
      }
    }
  }

  at = "drawn";
  for (int it = 0; it < 60000; ++it) {
    const int heads[] = {1, 2, 3, 8, 16, 32, 96};
    d.batch = rnd(0, 3) ? rnd(1, 70) : rnd(1, 600);
    d.kv_heads = heads[rnd(0, 6)];
    d.heads = d.kv_heads * rnd(1, 16);
    d.page_size = 16 << rnd(0, 4);
    d.table_pages = rnd(1, rnd(0, 1) ? 400 : 4000) * 16 / d.page_size + 1;
    d.window = rnd(0, 5) ? rnd(1, rnd(0, 1) ? 5000 : 30000) : 0;
    d.sinks = rnd(0, 1) ? 0 : rnd(0, 9) ? rnd(1, 100) : rnd(1, 3000);
    std::vector<int> lens(d.batch);
    const int kind = rnd(0, 2), base = rnd(0, capacity(&d) + 40);
    for (int& x : lens) x = kind == 0 ? base : kind == 1 ? rnd(0, capacity(&d) + 40) : std::max(0, base - rnd(0, 100));
    check(lens);
  }

  at = "rule";
  int64_t grown = 0;
  for (int it = 0; it < 60000; ++it) {
    const int batch = rnd(1, 100), room = rnd(1, 600), rows = std::max(batch, rnd(1, 1100)), low = 32 * rnd(4, 16), up_to = low * rnd(1, 2);
    std::vector<int64_t> n(batch);
    int64_t all_least = 0;
    for (auto& x : n) x = rnd(0, rnd(0, 4) ? 5000 : 200000), all_least += x > up_to ? (x + low - 1) / low : 1;
    const int64_t found = slices_found(n, (uint32_t)room, (uint32_t)rows, (uint32_t)up_to, (uint32_t)low);
    REQUIRE(found <= rows && found >= batch);
    grown += all_least > rows;
  }
  std::printf("host_paged_fp4_plan: ok, %lld calls, %lld cut, %lld lengths bounded by the plan, %lld with fewer rows than the least slices\n", (long long)calls, (long long)cut, (long long)bounded, (long long)grown);
  return calls > 100000 && cut > 100000 && bounded > 100000 && grown > 1000 ? 0 : 1;
}
