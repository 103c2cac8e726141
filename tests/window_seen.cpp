// win_seen against single pairs: prints "ok".
#include <cstdio>
#include <cstdlib>

#include "razor_window.h"

using namespace razor;

int main() {
  std::srand(1);
  auto rnd = [](int lo, int hi) { return lo + std::rand() % (hi - lo + 1); };
  for (int i = 0; i < 20000; ++i) {
    const int first = rnd(-20, 200), last = first + rnd(0, 60), window = rnd(0, 4) ? rnd(0, 150) : -1, n_sink = rnd(0, 3) ? rnd(0, 40) : 0;
    for (int n = 0; n < 280; ++n) {
      bool want = false;
      for (int m = first; m <= last; ++m) want |= n <= m && (n < n_sink || window < 0 || m - n < window);
      if (win_seen(n, first, last, window, n_sink) != want) {
        std::printf("key %d, queries %d .. %d, window %d, %d sinks: %d wanted\n", n, first, last, window, n_sink, want);
        return 1;
      }
    }
  }
  // the ends of the range
  if (win_seen((1LL << 30) - 1, (1 << 30) - 1, (1 << 30) - 1, 0, 0) || !win_seen(0, (1 << 30) - 1, (1 << 30) - 1, 1 << 30, 0)) return 1;
  std::printf("ok\n");
  return 0;
}
