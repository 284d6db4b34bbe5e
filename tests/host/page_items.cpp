// How the plan and the release of pages go through their items, up to the largest sizes that the calls take: every
// item of a launch once and none outside, and its request among up to 2^31 - 1 of them.
#include <stdio.h>

#include "paged.hpp"

// exclusive sums of a request's items: `per` each
struct Even {
  long long per;
  long long operator[](int r) const { return r * per; }
};

int main() {
  long long bad = 0, seen = 0;
  const int most = 0x7fffffff;
  for (int n : {0, 1, 255, 256, 8192, 1 << 20, most - (1 << 18) - 1, most - (1 << 18), most - (1 << 18) + 1, most - 1, most})
    for (int step : {1024, 4 * 256 * 256})
      for (int first : {0, 1, 1023}) {
        if (n > (1 << 25) && step == 1024) continue;  // (such a step is a launch of 8192 items at most)
        long long count = 0, last = first - (long long)step;
        laga::each_item(first, step, n, [&](int k) {
          if (k < 0 || k >= n || k != last + step) ++bad;
          last = k;
          if (++count > n) __builtin_trap();
        });
        if (count != (n > first ? ((long long)n - first + step - 1) / step : 0)) ++bad;
        seen += count;
      }
  for (int R : {1, 2, 3, 1000, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, (1 << 30) + 77, most - 1, most})
    for (int i = 0; i < 1000; ++i) {
      const int k = (int)((long long)i * (R - 1) / 999);
      if (laga::find_request(Even{1}, R, k) != k) ++bad;
    }
  for (int k : {0, 1, 65534, 65535, 2000000000}) {
    if (laga::find_request(Even{65535}, 32767, k) != k / 65535) ++bad;
  }
  printf("%lld items, %lld wrong\n", seen, bad);
  return bad != 0;
}
