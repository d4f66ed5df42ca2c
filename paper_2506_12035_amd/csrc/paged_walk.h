// Which tokens a block of rows over windows walks through (plain arithmetic, for the kernels
// and for the host).
#pragma once

#include <stdint.h>

namespace marche {

// Tiles of TK tokens, by their places in the walk: those that hold the sequence's first
// `sinks` tokens and, `jump` tiles further on, those from the earliest window's first token,
// `lo`, to the latest one's end, `hi`, a sequence's length at most.  lo has no such bound,
// as rows may stand past the length: a window that begins behind every token adds no
// tiles, and the jump ends with the last one.
template <int TK>
struct WindowWalk {
  int sink_tiles, jump, tiles;

  static constexpr int least(int a, int b) { return a < b ? a : b; }
  static constexpr int most(int a, int b) { return a > b ? a : b; }
  static constexpr int up(int tokens) { return (int)(((uint32_t)tokens + (TK - 1)) / TK); }

  static constexpr WindowWalk of(int lo, int hi, int sinks) {
    const int last = up(hi), kept = up(least(sinks, hi));
    const int from = least(most((int)((uint32_t)lo / TK), kept), last);
    return WindowWalk{kept, from - kept, kept + last - from};
  }
  // First token of a place.
  constexpr int key(int place) const { return TK * (place >= sink_tiles ? place + jump : place); }
};

// First token of part `part` (of 16) of a tile whose first token is key(place), or -1 where
// there is nothing to look up: places from `stop` on, whose keys may pass 32 bits, and
// tokens from `end` on.
template <typename Key>
constexpr int token_of(const Key &key, int place, int stop, int part, int end) {
  if (place >= stop) return -1;
  const int first = key(place);
  return 16 * part < end - first ? first + 16 * part : -1;
}

}  // namespace marche
