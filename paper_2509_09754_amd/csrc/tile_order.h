// The order in which a windowed decode step over pages takes a head's tiles, without device code: the kernel and a CPU test
// share it.
//
// With a window the rows that count lie together, and a run of tiles would have all of them or none.  The tiles of a head then take
// their places column by column of a matrix of kSpread rows, whose rows are taken kStep apart (place x is tile
// (kStep x % kSpread) * columns + x / kSpread, or none), so that every share has its part of the window, and (kSpread is odd)
// every wavefront of it.  24 windowed sequences: runs of tiles 51 us, 16 rows 47.7, several tiles a place (below) 42.4, 17 rows 39.8,
// rows 7 apart 38.3; the numbers were chosen on this one shape (7 heads a group, a window of 2048).
#pragma once

namespace lava {

constexpr int kTileKeys = 32;        // keys per MFMA tile

constexpr int kStep = 7;
constexpr int kSpread = 17;
constexpr int spread_columns(int tiles, bool spread) { return spread && tiles >= 4 * kSpread ? (tiles + kSpread - 1) / kSpread : 0; }
constexpr int places_of(int tiles, bool spread) {
  const int columns = spread_columns(tiles, spread);
  return columns > 0 ? columns * kSpread : tiles;
}
// With a window a place of the line is not one tile but 2, 4 or 8 of them: about as many as hold one that counts if the head's rows are spread
// over the sequence's positions (and no more than finding out costs).  An estimate: it moves cuts, not results.
constexpr int log_per_place(int q_pos, int window) {
  const long long seen = (long long)q_pos + 1;
  return seen >= 8ll * window ? 3 : seen >= 4ll * window ? 2 : seen >= 2ll * window ? 1 : 0;
}
constexpr int tile_at(int place, int columns) { return columns > 0 ? (place % kSpread * kStep % kSpread) * columns + place / kSpread : place; }
// First row of the tile at a place.  The last places of a head may be tiles it does not have, up to kSpread - 1 of them, and a
// head may have 2^31 - 16 rows: their first rows pass 2^31, so they are unsigned.
constexpr unsigned int row_at(int place, int columns) { return (unsigned int)tile_at(place, columns) * kTileKeys; }

}  // namespace lava
