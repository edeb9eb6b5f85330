// Driver for tests/test_row_range.py: "from to rows" each from stdin, "first count" each.
#include <cstdio>

#include "row_range.h"

int main() {
  int from, to, rows;
  while (scanf("%d %d %d", &from, &to, &rows) == 3) {
    const moe::RowRange r = moe::row_range(from, to, rows);
    printf("%d %d\n", r.first, r.count);
  }
  return 0;
}
