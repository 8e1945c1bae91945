// Which entries of a sequence's page table its tiles of 32 tokens read, on the host as on the device.
#ifndef QG_PAGES_H
#define QG_PAGES_H

#include "qg_position.h"

// Entries that a sequence of `keys` tokens has: no others are read
QG_POSITION_FN int qg_page_entries(int keys, int lgp) { return (keys + (1 << lgp) - 1) >> lgp; }

// The entry of a tile's tokens 0 .. 15 (half 0) or 16 .. 31 (half 1; one page has both but for pages of 16 tokens), or the last one:
// what a tile has behind the sequence's end is masked, wherever it was read.  The tile begins before the end.
QG_POSITION_FN int qg_page_entry(int t0, int half, int lgp, int entries) {
  const int index = (t0 + 16 * half) >> lgp;
  return index < entries ? index : entries - 1;
}

#endif
