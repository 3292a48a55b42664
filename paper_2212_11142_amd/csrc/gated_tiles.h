// Which tile a block of the gated block's kernels takes. (Nothing but arithmetic, for the device and for the host.)
#pragma once

namespace bgp {

// Tile of a block: neighbours in m share an XCD's cache for the n side, eight m tiles to a group.
struct Tile {
  int m, n;
};
constexpr Tile tile_of(unsigned block, unsigned blocks, int nm, int nn) {
  // blocks go round the 8 XCDs: each gets a run of tiles
  const unsigned per = blocks / 8, more = blocks % 8, x = block % 8;
  const unsigned i = x * per + (x < more ? x : more) + block / 8;
  constexpr unsigned kGroup = 8;
  const unsigned group = i / (kGroup * nn), in = i - group * kGroup * nn;
  const unsigned left = nm - group * kGroup, size = left < kGroup ? left : kGroup;
  return {(int)(group * kGroup + in % size), (int)(in / size)};
}

}  // namespace bgp
