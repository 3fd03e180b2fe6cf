// Tokens of append and reading launches, for tests/test_rows_tokens.py: every thread of a
// launch (its blocks' spare ones too, up to 255 past the end) gets a token of the
// launch's, and the launch's tokens each their own.  Built with traps on signed overflow.
#include <climits>
#include <cstdio>

#include "internal.h"

using namespace specmemo;

int main() {
  const int ends[] = {1, 2, 255, 256, 100000, INT_MAX - 1023, INT_MAX - 255, INT_MAX - 1, INT_MAX};
  for (const int tok1 : ends)
    for (const int n : {1, 2, 63, 255, 1024, 70000}) {
      if (n > tok1) continue;
      const int tok0 = tok1 - n;
      for (int i = 0; i < n + 256; ++i) {
        const RowsToken t = rows_token(tok0, tok1, i);
        if (t.on != (i < n) || t.tok < tok0 || t.tok >= tok1 || (t.on && t.tok - tok0 != i)) {
          std::printf("token %d of [%d, %d): %d, %d\n", i, tok0, tok1, t.tok, (int)t.on);
          return 1;
        }
      }
    }
  return 0;
}
