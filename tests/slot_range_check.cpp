// The slots that a weights' gradient takes (slot_range.hpp), near the largest slot
// numbers:
//
//   check LO HI PARTS STAGE
//
// prints 1 if the parts are ranges of [LO, HI) that follow one another, cover it,
// and begin at whole stages from LO on (the empty ones at HI), else 0;
//
//   check LO HI AHEAD
//
// prints the slot that lies AHEAD places behind LO.
#include <cstdint>
#include <cstdio>
#include <cstdlib>

#include "slot_range.hpp"

int main(int argc, char** argv) {
  if (argc == 4) {
    const unsigned ahead = static_cast<unsigned>(std::strtoul(argv[3], nullptr, 10));
    std::printf("%d\n", bitsmoe::slot_ahead(std::atoi(argv[1]), std::atoi(argv[2]), ahead));
    return 0;
  }
  if (argc != 5) return 2;
  const int lo = std::atoi(argv[1]), hi = std::atoi(argv[2]), parts = std::atoi(argv[3]), stage = std::atoi(argv[4]);
  int64_t at = lo;
  bool good = true;
  for (int p = 0; p < parts; ++p) {
    int a = lo, b = hi;
    bitsmoe::take_part(&a, &b, p, parts, stage);
    good = good && a == at && b >= a && b <= hi && (a == hi || (a - lo) % stage == 0);
    at = b;
  }
  std::printf("%d\n", good && at == hi);
  return 0;
}
