// Prints the tiles that X X^T, A A and B X of a stack of matrices take, one
// line a stack "batch rows cols" on the command line.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>

#include "mlkv_tiles.h"

int main(int argc, char** argv) {
  static const char* const names[] = {"64k", "64", "128", "192", "256"};
  const auto up = [](int64_t v) { return (v + mlkv::kOrthPad - 1) / mlkv::kOrthPad * mlkv::kOrthPad; };
  for (int i = 1; i + 2 < argc; i += 3) {
    const int64_t batch = atoll(argv[i]), rows = atoll(argv[i + 1]), cols = atoll(argv[i + 2]);
    const int64_t mp = up(std::min(rows, cols)), np = up(std::max(rows, cols));
    const auto name = [&](bool symmetric, int64_t k) {
      return names[(int)mlkv::orth_tile(mp, np, batch, symmetric, k)];
    };
    printf("%s %s %s\n", name(true, np), name(true, mp), name(false, mp));
  }
  return 0;
}
