// Where tokens lie in the paged cache, asked on the host: the library's own
// functions (csrc/serve.h), one answer a line.
//   row ENTRY PAGES HKV HEAD SHIFT SLOT | column T SHIFT TABLE_PAGES | len LEN CAPACITY
#include <cstdio>
#include <cstring>

#include "serve.h"

int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    long long v[6];
    const int n = !std::strcmp(what, "row") ? 6 : !std::strcmp(what, "column") ? 3 : 2;
    for (int i = 0; i < n; ++i)
      if (std::scanf("%lld", &v[i]) != 1) return 1;
    if (n == 6)
      std::printf("%lld\n", xattn::page_row((int)v[0], (int)v[1], (int)v[2], (int)v[3], (int)v[4],
                                            (int)v[5]));
    else if (n == 3)
      std::printf("%d\n", xattn::page_column(v[0], (int)v[1], (int)v[2]));
    else
      std::printf("%d\n", xattn::clamp_len((int)v[0], (int)v[1]));
  }
  return 0;
}
