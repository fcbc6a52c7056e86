// csrc/matrix.h: whether two matrices share a byte, against marking every byte.
#include <cstdio>
#include <vector>

#include "matrix.h"

int main() {
  uint32_t seed = 1;
  auto pick = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (uint32_t)n); };
  long shared = 0, n = 0;
  for (int k = 0; k < 400000; ++k, ++n) {
    oseq::Place p[2];
    std::vector<char> mark(4096, 0);
    bool want = false;
    for (int i = 0; i < 2; ++i) {
      p[i].width = 1 + pick(12);
      p[i].pitch = k % 3 && i ? p[0].pitch : p[i].width + pick(30);
      if (p[i].pitch < p[i].width) p[i].width = p[i].pitch;
      p[i].rows = 1 + pick(9);
      p[i].at = 4096 + pick(200);
      for (int r = 0; r < p[i].rows; ++r)
        for (int c = 0; c < p[i].width; ++c) {
          char& m = mark[p[i].at - 4096 + r * p[i].pitch + c];
          want |= i == 1 && m;
          if (i == 0) m = 1;
        }
    }
    shared += want;
    if (oseq::overlap(p[0], p[1]) != want || oseq::overlap(p[1], p[0]) != want) { std::printf("case %d: want %d\n", k, (int)want); return 1; }
  }
  std::printf("ok %ld, %ld shared\n", n, shared);
}
