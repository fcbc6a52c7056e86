// csrc/parts.h: the parts of a reduction lie one behind the other from 0 to K, for every K the layers admit (built with UBSan: nothing wraps).
#include <cstdio>

#include "parts.h"

static bool whole(int K, int wanted) {
  const oseq::Parts p = oseq::parts_of(K, wanted);
  if (p.count < 1 || p.count > wanted || p.size % 64) return false;
  int at = 0;
  for (int i = 0; i < p.count; ++i) {
    if (p.first(i) != at || p.end(i) <= at || p.end(i) - at > p.size) return false;
    at = p.end(i);
  }
  return at == K;
}

int main() {
  long n = 0;
  for (int wanted = 1; wanted <= 32; ++wanted) {
    for (int K = 1; K <= 5000; ++K, ++n)
      if (!whole(K, wanted)) { std::printf("K %d in %d\n", K, wanted); return 1; }
    for (int K = 0x7fffff00; K > 0x7fffff00 - 5000; --K, ++n)
      if (!whole(K, wanted)) { std::printf("K %d in %d\n", K, wanted); return 1; }
    for (int64_t K = 5000; K <= 0x7fffff00; K += K / 3 + 1, ++n)
      if (!whole((int)K, wanted)) { std::printf("K %d in %d\n", (int)K, wanted); return 1; }
  }
  std::printf("ok %ld\n", n);
}
