// narrow_floor (floors.hpp) on the CPU, over waves of 64 numbers in the order that the kernels give to logits:
//   1. of logits that differ, a number is found that c to c + c / 4 + 1 of them reach, whatever offset and spread
//      the logits have and however far one of them stands out, in about as many steps;
//   2. of equal ones, one is found that c reach and that cannot be raised, unless few enough reach it.
// Prints "OK" and exits 0 when every check holds.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "floors.hpp"

namespace {

int g_fail = 0;

uint32_t ordered(float x) {
  uint32_t b;
  std::memcpy(&b, &x, 4);
  return b ^ ((int32_t)b < 0 ? ~0u : 0x80000000u);
}

struct Found {
  int reach, steps;
  bool raised;  // the next number is reached by fewer than c
};

Found search(const std::vector<uint32_t>& u, int c) {
  const auto count = [&](uint32_t m) { return (int)std::count_if(u.begin(), u.end(), [=](uint32_t x) { return x >= m; }); };
  int steps = 0;
  const uint32_t f = spp::narrow_floor(*std::min_element(u.begin(), u.end()), *std::max_element(u.begin(), u.end()),
                                       c, [&](uint32_t m) { return ++steps, count(m); });
  return Found{count(f), steps, count(f + 1) < c};
}

void expect(bool ok, const char* what, double offset, double spread, int c, const Found& f) {
  if (ok) return;
  if (++g_fail < 20)
    std::fprintf(stderr, "%s: offset %g, spread %g: of 64 numbers %d reach what %d are to reach, after %d steps\n", what,
                 offset, spread, f.reach, c, f.steps);
}

}  // namespace

int main() {
  std::mt19937 rng(7);
  std::normal_distribution<double> normal;
  for (double spread : {2.0, 0.05, 40.0})
    for (double offset : {0.0, 300.0, -300.0, 1000.0, -1000.0, 12.0})
      for (int c : {2, 4, 5, 13, 16, 20, 33, 63, 64}) {
        long total = 0;
        for (int k = 0; k < 40; ++k) {
          std::vector<uint32_t> u;
          // the largest of 160 each, as the merge's threads have them
          while (u.size() < 64) {
            float most = -INFINITY;
            for (int i = 0; i < 160; ++i) most = std::max(most, (float)(normal(rng) * spread + offset));
            if (u.size() == 5) most += (float)(spread * (k % 4) * 20);  // one that stands out
            if (std::find(u.begin(), u.end(), ordered(most)) == u.end()) u.push_back(ordered(most));
          }
          const Found f = search(u, c);
          expect(f.reach >= c && f.reach <= c + c / 4 + 1, "differing", offset, spread, c, f);
          total += f.steps;
        }
        if (total > 16 * 40) expect(false, "steps", offset, spread, c, Found{0, (int)(total / 40), false});
      }
  for (int values : {1, 2, 3, 10})
    for (double offset : {0.0, 500.0})
      for (int c : {2, 7, 16, 64})
        for (int k = 0; k < 100; ++k) {
          std::vector<uint32_t> u(64);
          for (auto& x : u) x = ordered((float)(offset + (double)(rng() % values) - 1));
          const Found f = search(u, c);
          expect(f.reach >= c && (f.reach <= c + c / 4 + 1 || f.raised) && f.steps <= 40, "equal", offset, values, c, f);
        }
  const std::vector<uint32_t> ends{1u, 0xFFFFFFFEu, 0x80000000u, 0x7FFFFFFFu};
  for (int c = 1; c <= 4; ++c) expect(search(ends, c).reach >= c, "ends", 0, 0, c, search(ends, c));
  if (g_fail) return 1;
  std::printf("OK\n");
  return 0;
}
