// Which of an expert's slots a part of the weights' gradient sums, and which are
// asked for ahead.  Plain integer rules without device code, so that they can be
// checked on the host: slot numbers go up to 2^31 - 257, and what lies a part or
// eight stages behind the last one passes 31 bits.
#pragma once

namespace bitsmoe {

// [lo, hi) to its `part`th of `parts`: as many stages of `stage` slots each, the
// last ones fewer or none.  (By what is left, not by where a part would end:
// 256 parts of 2^31 - 16383 slots end at 2^31.)
constexpr void take_part(int* lo, int* hi, int part, int parts, int stage) {
  const unsigned slots = *hi - *lo;
  const unsigned each = ((slots + stage - 1) / stage + parts - 1) / parts * stage;
  const unsigned skip = part * each < slots ? part * each : slots, left = slots - skip;
  *lo += static_cast<int>(skip);
  *hi = *lo + static_cast<int>(each < left ? each : left);
}

// The slot `ahead` places behind lo, or -1 if it is not one of [lo, hi).
constexpr int slot_ahead(int lo, int hi, unsigned ahead) {
  return ahead < static_cast<unsigned>(hi - lo) ? lo + static_cast<int>(ahead) : -1;
}

}  // namespace bitsmoe
