// Driver for tests/test_row_grid.py: the grid for numbers of workgroups read from stdin, "x y" each.
#include <cstdio>

#include "row_grid.h"

int main() {
  long long groups;
  while (scanf("%lld", &groups) == 1) {
    const moe::RowGrid g = moe::row_grid(groups);
    printf("%u %u\n", g.x, g.y);
  }
  return 0;
}
