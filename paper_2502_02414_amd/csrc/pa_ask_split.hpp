// How attention over few states is split over blocks (host code, no HIP headers), and
// how far a kernel's count of rows may run past a tensor's last one.
#pragma once

#include <algorithm>
#include <cstdint>

namespace pa {

// Virtual rows and states are counted in 32 bits: a call has at most kMostRows of either,
// and no loop adds more than kRowsAhead to a row that there is.
constexpr int64_t kRowsAhead = 1 << 21, kMostRows = 0x7fffffff - kRowsAhead;

// Blocks of a request (P), groups of heads, how many waves of a block share a head (subs),
// and a block's waves.  Forward: whole rounds of the blocks that are resident, each wave with
// some 16 tiles (us, of 64 states of 8 heads of 32: 100,000 queries 27 where blocks of two
// tiles took 40, a million 240 and, in 1953 blocks, 252; 300,000 of 4 heads of 64 67 and 108).
// Backward: a block per CU, since each leaves a record of all states' gradients.
struct FewSplit {
  int P, groups, subs, waves;
  // rows from one of a wave's tiles of 32 to its next
  int64_t step() const { return (int64_t)32 * subs * P; }
};
inline FewSplit few_split(int64_t Nq, int R, int Hq, int Hkv, int D, int64_t max_k, bool bwd) {
  FewSplit s;
  s.waves = bwd && D > 32 && max_k > 32 ? 4 : 8;
  const int heads = Hkv < s.waves ? Hkv : s.waves;
  s.groups = (Hkv + heads - 1) / heads;
  s.subs = s.waves / heads;
  const int64_t n = Nq * (Hq / Hkv) / R, each = (int64_t)R * s.groups;
  int64_t P = 256 / each, least = 64 * s.subs;
  if (!bwd) {
    const int64_t resident = D > 32 && max_k > 32 ? 256 : 512, rows = n * each / s.subs;
    const int64_t rounds = (rows / 256 / resident + 1) / 2;
    P = (rounds ? rounds * resident : std::min(resident, std::max<int64_t>(256, rows / 128))) / each;
    least = 32 * s.subs;
  }
  if (P > n / least) P = n / least;
  // (each wave has more than 16 tiles then)
  P = std::min(P, kRowsAhead / (32 * s.subs));
  s.P = P < 1 ? 1 : (int)P;
  return s;
}

}  // namespace pa
