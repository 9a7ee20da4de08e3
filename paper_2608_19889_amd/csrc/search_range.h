// The range of sort keys in which a search over histograms looks for its border.
#pragma once
#include <cstdint>

namespace axon {

constexpr int BINS = 2048;

// Keys lo .. hi, in BINS bins of 2^shift() keys each from lo on, a search's entries being
// the bins from the last one down.
struct KeyRange {
  uint32_t lo, hi;
  constexpr int shift() const {
    int s = 0;
    while ((hi - lo) >> s >= BINS) ++s;
    return s;
  }
  // The keys of entry ``at``.  Smaller than the range, or one key, so that a search ends
  // whatever it is given: false, and the range as it was, where ``at`` is none of its
  // entries (a search that found nothing gives -1).
  constexpr bool narrow(int at) {
    const int s = shift();
    if (at < 0 || at >= BINS) return false;
    const uint32_t bin = BINS - 1 - at;
    if (bin > (hi - lo) >> s) return false;
    lo += bin << s;
    const uint32_t rest = hi - lo, width = (1u << s) - 1;
    hi = lo + (rest < width ? rest : width);
    return true;
  }
};

}  // namespace axon
