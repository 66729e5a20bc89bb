// Asks the serving calls' own dispatch rules (csrc/serve.h) on the host.
//   workers ROWS TWO_TILES | one answer a line
#include <cstdio>
#include <cstring>

#include "serve.h"

int main() {
  char what[16];
  int a, b;
  while (std::scanf("%15s %d %d", what, &a, &b) == 3) {
    if (std::strcmp(what, "workers") != 0) return 1;
    std::printf("%d\n", xattn::decode_workers(a, b != 0));
  }
  return 0;
}
