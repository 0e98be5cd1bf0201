// rows_share against a count of bytes, at random places, lengths and steps.
#include <cstdio>
#include <random>
#include <vector>

#include "overlap.h"

using grpo::ByteRows;
using grpo::rows_share;

int main() {
  std::mt19937 rng(5);
  auto any = [&](int lo, int hi) { return (int)(lo + rng() % (unsigned)(hi - lo + 1)); };
  long met = 0, apart = 0;
  for (int k = 0; k < 400000; ++k) {
    const int esz = any(0, 1) ? 2 : 4, same = any(0, 1), cols[2] = {any(1, 9), any(1, 9)}, rows[2] = {any(1, 7), any(1, 7)};
    int ld[2] = {cols[0] + any(0, 12), cols[1] + any(0, 12)};
    if (same) ld[0] = ld[1] = std::max(ld[0], ld[1]);
    const int at[2] = {any(0, 400), any(0, 400)};
    std::vector<char> hit(2000, 0);
    for (int i = 0; i < rows[0]; ++i)
      for (int c = 0; c < cols[0] * esz; ++c) hit[at[0] + i * ld[0] * esz + c] = 1;
    bool want = false;
    for (int i = 0; i < rows[1]; ++i)
      for (int c = 0; c < cols[1] * esz; ++c) want |= hit[at[1] + i * ld[1] * esz + c] != 0;
    const ByteRows a((void*)(uintptr_t)(0x1000 + at[0]), rows[0], cols[0], ld[0], esz),
        b((void*)(uintptr_t)(0x1000 + at[1]), rows[1], cols[1], ld[1], esz);
    if (rows_share(a, b) != want || rows_share(b, a) != want) {
      printf("at %d: %d rows of %d, %d apart; at %d: %d of %d, %d apart; %d bytes: not %d\n", at[0], rows[0], cols[0], ld[0],
             at[1], rows[1], cols[1], ld[1], esz, want);
      return 1;
    }
    (want ? met : apart) += 1;
  }
  // the ends of the ranges, where products of sizes pass 64 bits
  const int64_t most = 8388352, big = INT64_MAX;
  const ByteRows far((void*)0x1000, most, most, big, 4), one((void*)0x2000, 1, 1, big, 4), none(nullptr, 5, 5, 5, 2);
  if (!rows_share(far, one) || rows_share(far, none) || rows_share(none, none)) return 2;
  if (met < 20000 || apart < 20000) return 3;
  printf("rows share ok\n");
  return 0;
}
