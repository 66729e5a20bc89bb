// Asks the library's own rule (csrc/serve.h) whether two arrays of vectors meet.
//   APART BATCH_STRIDE HEAD_STRIDE TOKEN_STRIDE BATCH HEADS TOKENS | one answer a line
#include <cstdio>

#include "serve.h"

int main() {
  long long v[7];
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld", v, v + 1, v + 2, v + 3, v + 4, v + 5,
                    v + 6) == 7)
    std::printf("%d\n", xattn::vectors_meet(v[0], xattn::Strides{v[1], v[2], v[3]}, (int)v[4],
                                            (int)v[5], (int)v[6]));
  return 0;
}
