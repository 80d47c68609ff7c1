// With "plan F32 CUS T H F": tile, splits and launch of the forward and of the backward, and whether their parts of the workspace lie one
// behind the other; F32 1 or 0.  With "steps K STEP A B": whole_steps() of csrc/glu_plan.h; with "reads MOST_ROW MOST_K": checks, for every row of up to MOST_ROW
// elements, every k up to MOST_K and steps of 32 and 64, that no piece of a whole step ends behind the operand, and prints how many
// were looked at, and the first that does.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../paper_2210_10246_amd/csrc/glu_plan.h"

namespace {

// As test_gpu_glu_plans.py writes them.
void print(const tempo::Plan& p, bool padded) {
  const char* edges[] = {"256", "128", "64", "few 16", "few 64", "few 128"};
  const int i = static_cast<int>(p.size);
  std::printf("%s%s", i > 2 ? "" : padded ? "P" : p.aligned ? "A" : "R", edges[i]);
}

void plans(int64_t T, int64_t H, int64_t F, tempo_dtype dt, int cus) {
  const tempo::ForwardPlan f(T, H, F, dt, cus);
  print(f.plan, f.padded);
  std::printf("%s | ", f.plan.splits > 1 ? "+" : "");
  const tempo::BackwardPlan b(T, H, F, dt, cus);
  print(b.plans[0], b.padded);
  std::printf("%s%s", b.plans[0].splits > 1 ? " dx+" : "", b.plans[1].splits > 1 ? " dw+" : "");
  // parts of k cover it, and every region of the workspace is as long as what goes into it
  auto covers = [](const tempo::Plan& p, int64_t K, int step) { return int64_t{p.splits} * p.steps * step >= K; };
  auto step = [&](const tempo::Plan& p) { return dt == TEMPO_F32 || (p.aligned && p.size < tempo::Size::kSmall) ? 32 : 64; };
  auto sums = [](const tempo::Plan& p, int64_t M, int64_t N) { return p.splits > 1 ? size_t(p.splits) * M * N * 4 : 0; };
  const size_t copies = size_t(T + 2 * F) * f.H_pad * 2, dgu = b.F2_pad != 2 * F ? size_t(T) * b.F2_pad * 2 : 0;
  const bool ok = covers(f.plan, H, step(f.plan)) && covers(b.plans[0], 2 * F, step(b.plans[0])) &&
                  covers(b.plans[1], T, step(b.plans[1])) && f.x_at >= sums(f.plan, T, 2 * F) &&
                  f.bytes == f.x_at + (f.padded ? copies : 0) && b.dx_bytes >= sums(b.plans[0], T, H) &&
                  b.dgu_at >= b.dx_bytes + sums(b.plans[1], 2 * F, H) && b.x_at == b.dgu_at + (b.padded ? dgu : 0) &&
                  b.bytes == b.x_at + (b.padded && b.H_pad != H ? copies : 0) && f.x_at % 16 + b.dx_bytes % 16 + b.dgu_at % 16 == 0 &&
                  b.plans[0].aligned == b.plans[1].aligned && b.plans[0].size == b.plans[1].size;
  std::printf(" | %s\n", ok ? "fits" : "does not fit");
}

}  // namespace

int main(int argc, char** argv) {
  auto arg = [&](int i) { return i < argc ? std::atoi(argv[i]) : 0; };
  if (argc > 3 && std::strcmp(argv[1], "plan") == 0) {
    for (int i = 4; i + 2 < argc; i += 3)
      plans(arg(i), arg(i + 1), arg(i + 2), arg(2) ? TEMPO_F32 : TEMPO_BF16, arg(3));
    return 0;
  }
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
