"""How attention over few states splits its rows over blocks (csrc/pa_ask_split.hpp),
compiled for the CPU: the kernels count rows in 32 bits, so that a wave's step from one
of its tiles to the next has to stay within what the calls leave below 2^31."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2502_02414_amd", "csrc")

HARNESS = r"""
#include <cstdio>

#include "pa_ask_split.hpp"

int main() {
  static_assert(pa::kMostRows + pa::kRowsAhead <= 0x7fffffff, "counted in 32 bits");
  int bad = 0;
  const int64_t rows[] = {0, 1, 63, 64, 1000, 1000003, 33554432, 33554433, 268435456, 1073741823,
                          2021000000, 2100000000, pa::kMostRows - 1, pa::kMostRows};
  for (int64_t all : rows)
    for (int Hkv : {1, 2, 3, 4, 5, 8, 9, 16, 64, 512, 4096})
      for (int G : {1, 2, 3, 8, 64, 4096})
        for (int R : {1, 2, 7, 300, 1 << 20})
          for (int D : {8, 32, 64})
            for (int max_k : {1, 32, 33, 64})
              for (int bwd = 0; bwd < 2; ++bwd) {
                if ((int64_t)Hkv * G > 4096) continue;
                const pa::FewSplit s = pa::few_split(all / G, R, Hkv * G, Hkv, D, max_k, bwd);
                // the last row of a request of all rows and the one that is asked for
                // behind it; the grid's threads; every head has a wave
                const int64_t n = all / G * G, last = n ? n - 1 : 0;
                const int64_t threads = (int64_t)R * s.P * 64 * s.waves;
                if (s.P < 1 || s.subs < 1 || s.step() > pa::kRowsAhead || last + s.step() > 0x7fffffff ||
                    threads > 0xffffffffll || s.groups * (s.waves / s.subs) < Hkv) {
                  if (++bad <= 10)
                    std::printf("rows %lld Hkv %d G %d R %d D %d max_k %d backward %d: P %d step %lld\n",
                                (long long)all, Hkv, G, R, D, max_k, bwd, s.P, (long long)s.step());
                }
              }
  std::printf("%d refused\n", bad);
  return bad != 0;
}
"""


def test_a_step_past_the_last_row_stays_in_32_bits(tmp_path):
    src, exe = tmp_path / "split.cpp", tmp_path / "split"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", CSRC, str(src), "-o",
                    str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
