// How the paged attention shares out its tiles: every tile of every row belongs to one worker;
// of a row that several workers share, each leaves its partial in a place that no other share
// uses; and the join, which counts a row's workers from its tiles alone, finds those partials.
#include <stdio.h>

#include <vector>

#include "paged.hpp"

int main() {
  long long shares = 0, bad = 0;
  unsigned seed = 1;
  auto rnd = [&](unsigned n) { return (seed = seed * 1664525u + 1013904223u) / 65536u % n; };
  for (int heads : {1, 16, 33, 128, 129, 1000})
    for (int d_c : {32, 128, 256, 512, 1024})
      for (int es : {2, 4}) {
        const laga::PagedPlan p = laga::paged_plan(heads, d_c, 64, es);
        if (p.workers < 8 || p.workers % 8 || p.head_blocks * p.heads_per_wg < heads ||
            (p.head_blocks - 1) * p.heads_per_wg >= heads || p.groups < 0)
          ++bad;
        for (int rows : {1, 2, 7, 64, 300, 5000})
          for (int longest : {0, 1, 2, 40, 700, 9000}) {
            std::vector<long long> before(rows + 1, 0);
            std::vector<int> seen(rows);
            long long tiles = 0;
            int live = 0;
            for (int t = 0; t < rows; ++t) {
              const int visible = rnd(4) == 0 ? 0 : longest ? (int)rnd(32 * longest) + 1 : 0;
              seen[t] = visible;
              tiles += laga::tiles_of(visible);
              live += visible > 0;
            }
            const laga::Shares sh = laga::shares_of((int)tiles, live, p.workers, p.groups);
            for (int t = 0; t < rows; ++t) before[t + 1] = before[t] + laga::units_of(seen[t], sh.cost);
            const int total = (int)before[rows], per = sh.per;
            if (total != sh.total) ++bad;
            if ((long long)per * sh.workers < total || per < 1 || sh.workers > p.workers || sh.workers % 8) ++bad;
            // with few tiles every group of heads has its workers among the workgroups
            if (sh.groups && (sh.groups * 32 < p.heads_per_wg || sh.workers * sh.groups > p.workers)) ++bad;
            std::vector<int> place(2 * p.workers, -1), partials(rows, 0);
            long long done = 0;
            for (int w = 0; w < sh.workers; ++w) {
              const long long start = (long long)w * per, end = start + per < total ? start + per : total;
              for (int t = 0; t < rows; ++t) {
                const long long first = before[t] + sh.cost, a = first > start ? first : start, b = before[t + 1] < end ? before[t + 1] : end;
                if (a >= b) continue;
                ++shares;
                done += b - a;
                if (a == first && b == before[t + 1]) continue;  // whole
                const int at = laga::partial_place(w, per, (int)first);
                if (at < 0 || at >= 2 * p.workers || place[at] >= 0) ++bad;
                else place[at] = t;
                ++partials[t];
              }
            }
            if (done != tiles) ++bad;
            for (int t = 0; t < rows; ++t) {
              if (before[t] == before[t + 1]) continue;
              const int first = (int)before[t] + sh.cost, w0 = first / per, w1 = (int)((before[t + 1] - 1) / per);
              if (partials[t] != (w0 == w1 ? 0 : w1 - w0 + 1)) ++bad;
              for (int w = w0; w <= w1 && w1 > w0; ++w)
                if (place[laga::partial_place(w, per, first)] != t) ++bad;
            }
          }
      }
  // division by the page size
  for (int page : {1, 2, 3, 7, 16, 31, 48, 64, 200, 1000, 4096, 65535, 1 << 20, (1 << 29) + 1, 1 << 30}) {
    uint32_t magic, shift;
    laga::page_division(page, &magic, &shift);
    for (int i = 0; i < 20000; ++i) {
      const long long q = rnd(65536) * 65536ll + rnd(65536), k = i % 3 ? q % 0x7fffffff : q / page % (0x7fffffff / page) * page;
      for (long long key : {k, k - 1, k + page - 1, 0x7fffffffll - i})
        if (key >= 0 && key <= 0x7fffffff && (long long)((uint64_t)(uint32_t)key * magic >> shift) != key / page) ++bad;
    }
  }
  printf("%lld shares, %lld wrong\n", shares, bad);
  return bad != 0;
}
