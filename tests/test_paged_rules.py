"""How single-token attention over pages divides its work (compiled with the host compiler; no GPU): every tile of every sequence in exactly one range, every
part in a place of its own within the workspace, whatever the lengths; and which way of dividing a launch takes."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = '''#include <cstdio>
#include <cstdlib>
#include <vector>
#include <set>
#include "paged_rules.hpp"
static uint64_t state = 88172645463325252ull;
static int rnd(int n) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return (int)(state % (uint64_t)n); }
#define NEED(x) do { if (!(x)) { printf("%s: B %d ranges %d total %d\\n", #x, B, ranges, total); return 1; } } while (0)
int main() {
  for (int round = 0; round < 4000; ++round) {
    const int B = 1 + rnd(round % 3 ? 9 : 300), ranges = 1 + rnd(round % 2 ? 2048 : 40), most = 1 + rnd(round % 5 ? 20 : 700);
    std::vector<int> starts(B + 1, 0);
    for (int b = 0; b < B; ++b) starts[b + 1] = starts[b] + (rnd(4) ? rnd(most) : 0);
    const int total = starts[B], per = paged_tiles_of_range(total, ranges);
    NEED((long)per * ranges >= total && per >= 1);
    std::set<int> places;
    std::vector<char> seen(total, 0);
    for (int r = 0; r < ranges; ++r)                               // as the ranges take them
      for (int x = r * per; x < std::min(total, (r + 1) * per);) {
        int b = 0;
        while (starts[b + 1] <= x) ++b;
        const int stop = std::min({starts[b + 1], total, (r + 1) * per});
        const int first = paged_first_range(starts[b], per), last = paged_last_range(starts[b + 1], per);
        NEED(r >= first && r <= last);                             // as the parts are joined
        NEED((first == last) == (x == starts[b] && stop == starts[b + 1]));
        NEED(places.insert(r + b).second && r + b < ranges + B);
        for (; x < stop; ++x) NEED(!seen[x]++);
      }
    for (char c : seen) NEED(c == 1);
  }
  // the rule: bounds that the kernels rely on
  for (int B : {1, 2, 7, 64, 256, 257, 1024, 1025, 65535})
    for (int Hkv : {1, 2, 8, 40, 300, 65535})
      for (int G : {1, 4, 16, 17, 64})
        for (int n : {1, 511, 512, 513, 1024, 1025, 4096, 131072, 1 << 30}) {
          const int H = Hkv * G, total = 0;
          const bool fp32 = B & 1;
          const PagedSplit s = paged_split(B, H, Hkv, 128 << (B & 1), fp32, n);
          const int ranges = s.ranges, units = s.units;
          NEED((s.rows == 16 || (s.rows == 32 && !fp32 && G > 16)) && units == Hkv * ((G + s.rows - 1) / s.rows));
          NEED(ranges >= 0 && ranges <= 256 * PAGED_WAVES);
          NEED(ranges == 0 || ((long)B * (n / 16 + 1) < 1l << 30 && B <= 1024 && (long)ranges * units <= std::max(256l * PAGED_WAVES, (long)units)));
          NEED(n > 768 || ranges == 0);
          NEED(s.team || ranges == 0 || units >= 8);
        }
  const PagedSplit a = paged_split(1, 32, 8, 256, false, 4096), b = paged_split(1, 64, 8, 128, false, 131072), c = paged_split(64, 32, 8, 128, false, 2048),
                   d = paged_split(64, 32, 8, 256, false, 2048), e = paged_split(19, 24, 1, 128, false, 103066), f = paged_split(4, 24, 1, 256, false, 700);
  printf("%d %d  %d %d  %d %d  %d  %d %d %d  %d %d\\n", a.ranges, a.team, b.ranges, b.team, c.ranges, c.team, d.ranges, e.rows, e.ranges, e.team, f.rows, f.units);
  return 0;
}
'''


def test_division_of_tiles_and_the_rule(tmp_path):
    (tmp_path / "m.cpp").write_text(PROGRAM)
    inc = os.path.join(ROOT, "paper_2503_01840_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O2", "-I", inc, str(tmp_path / "m.cpp"), "-o", str(tmp_path / "m")], check=True)
    r = subprocess.run([str(tmp_path / "m")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert r.stdout.split() == "32 1 256 0 256 0 0 32 256 1 16 2".split()
