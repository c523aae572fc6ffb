// The number of parts that prefill_join_kernel takes from a workspace word, for any contents of that word.  Built and run by
// tests/test_operators_cpu.py.
#include <climits>
#include <cstdio>

#include "partition.h"

int main() {
  const int words[] = {INT_MIN, -1, 0, 1, 2, 3, 17, 36, 37, 38, 148, 1 << 20, 0x3f800000, 0x7f7f7f7f, INT_MAX};
  for (int splits = 2; splits <= 148; ++splits)
    for (int word : words) {
      const int parts = pdattn::join_parts(word, splits);
      if (parts < 0 || parts > splits || (word >= 0 && word <= splits && parts != word)) {
        std::fprintf(stderr, "join_parts(%d, %d) = %d\n", word, splits, parts);
        return 1;
      }
    }
  std::puts("join_parts_check: ok");
  return 0;
}
