// With "steps K STEP A B": whole_steps() of csrc/glu_plan.h; with "reads MOST_ROW MOST_K": checks, for every row of up to MOST_ROW
// elements, every k up to MOST_K and steps of 32 and 64, that no piece of a whole step ends behind the operand, and prints how many
// were looked at, and the first that does.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../paper_2210_10246_amd/csrc/glu_plan.h"

int main(int argc, char** argv) {
  auto arg = [&](int i) { return i < argc ? std::atoi(argv[i]) : 0; };
  if (argc == 6 && std::strcmp(argv[1], "steps") == 0) {
    std::printf("%d\n", tempo::whole_steps(arg(2), arg(3), arg(4), arg(5)));
    return 0;
  }
  long long pieces = 0;
  for (int n = 1; n <= arg(2); ++n)
    for (int k = 0; k <= arg(3); ++k)
      for (int step = 32; step <= 64; step += 32) {
        const int whole = tempo::whole_steps(k, step, n, 0);
        if (whole * step > k || whole != tempo::whole_steps(k, step, 0, n) || whole > tempo::whole_steps(k, step, 0, 0)) return 1;
        for (int line = 0; line < whole * step; ++line)      // as the kernel places them: tiles end behind a row of few elements
          for (int at = 0; at < 256; at += 8, ++pieces)
            if (static_cast<long long>(line) * n + std::min(at, (n - 1) & ~7) + 8 > static_cast<long long>(k) * n) {
              std::printf("%lld %d %d %d\n", pieces, n, k, step);
              return 0;
            }
      }
  std::printf("%lld\n", pieces);
}
