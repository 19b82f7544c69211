// Host check of the chunks that the layer norm's launches cut rows into (csrc/internal.h): they cover every row
// once, there are no more of them than asked for, and none is empty, up to the largest number of rows. Prints the
// number of violations and exits non-zero if there is any.
#include <cstdio>
#include <initializer_list>

#include "internal.h"

int main() {
  long cases = 0, bad = 0;
  const int64_t last = (int64_t(1) << 31) - 1;
  const auto check = [&](int64_t S, int64_t most) {
    const refadapt::RowChunks c = refadapt::row_chunks((int32_t)S, most);
    const int64_t per = c.rows_per, n = c.count;
    ++cases;
    const bool covered = n * per >= S && (n == 0 || (n - 1) * per < S) && (S > 0) == (n > 0);
    if (per < 1 || n < 0 || n > (most < 1 ? 1 : most) || !covered)
      if (bad++ < 10)
        std::printf("violation: %lld rows, at most %lld chunks: %lld of %lld\n", (long long)S, (long long)most,
                    (long long)n, (long long)per);
  };
  for (int64_t S = 0; S < 700; ++S)
    for (int64_t most = 0; most < 700; ++most) check(S, most);
  for (int64_t most : {1, 2, 7, 256, 512, 1000, 1024, 2048, 1 << 20, 1 << 24}) {
    for (int64_t d = 0; d < 3000; ++d) check(last - d, most);
    for (int64_t S = 1; S <= last; S = S * 3 / 2 + 1) check(S, most);
  }
  std::printf("%ld cases, violations %ld\n", cases, bad);
  return bad != 0;
}
