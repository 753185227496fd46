// The single elements of a row of logits (ops.h: row_edge): over every head, rows down to
// one element and up to the longest, the workgroup's threads cover exactly the
// elements outside the whole pieces, each once, and no other.
#include <stdint.h>
#include <stdio.h>

#include "ops.h"

int main() {
  int failures = 0;
  const int kMost = 0x7fffffff;
  for (int n = 4; n <= 8; n += 4)
    for (int lead = 0; lead < n; ++lead)
      for (int k = 0; k < 200; ++k) {
        const int V = k < 100 ? k + 1 : kMost - (k - 100);
        const int head = lead < V ? lead : V, full = (V - head) / n;
        const int64_t end = head + (int64_t)full * n;
        int64_t covered = 0;
        for (int t = 0; t < 1024; ++t) {
          const int64_t i = fp8q::row_edge(t, V, head, full, n);
          if (i == -1) continue;
          ++covered;
          if (i < 0 || i >= V || (i >= head && i < end)) {
            printf("V %d head %d pieces of %d: thread %d has element %lld\n", V, head, n, t, (long long)i);
            ++failures;
          }
          if (i != (t < head ? t : end + (t - 32))) ++failures;
        }
        if (covered != V - full * (int64_t)n) ++failures;
      }
  printf("%d failures\n", failures);
  return failures != 0;
}
