// Which keys a query of a windowed causal attention sees, by position: plain
// arithmetic, for the host as for the device.
#pragma once
#include <stdint.h>

namespace tlf {

// The keys that the query at position p of a sequence sees, in order: the sinks ahead
// of the window, then those from `near` to p.  window is INT32_MAX where there is none.
// A query before the first key (p < 0) sees none; its p - window would leave 32 bits.
struct VisibleKeys {
  int near, sinks, count;
  constexpr VisibleKeys(int p, int window, int most_sinks)
      : near(p < window ? 0 : p - window + 1),
        sinks(p < 0 ? 0 : most_sinks < near ? most_sinks : near),
        count(p < 0 ? 0 : sinks + (p - near) + 1) {}
  constexpr int operator[](int i) const { return i < sinks ? i : near + (i - sinks); }
};

}  // namespace tlf
