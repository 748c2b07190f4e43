// Paged attention: the units in one order (a list's copies one after another), each at a place, in
// tiles, that follows from its list's first row alone; chunks of equal length are cut from it.
// Integers alone, which a host's compiler takes as well.
#pragma once

#include <stdint.h>

namespace certkv {

constexpr uint32_t kPgMinTiles = 4;    // shortest chunk, and the unit of its length
constexpr uint32_t kPgMaxTiles = 512;  // longest, unless partials are short
// Places are counted in 32 bits, of which the sums of two need all: tiles of all units must be fewer.
// (The lists' rows are the caller's on the device, and lists that share pages may have more than the
// pool holds.)
constexpr uint64_t kPgMostTiles = 0x7fffffff;

__host__ __device__ __forceinline__ uint32_t pg_up(int64_t rows) {
  return (uint32_t)((uint64_t)(rows + 31) >> 5);
}
// The first tile of list r, for copies = 1.
__host__ __device__ __forceinline__ uint32_t pg_place(int64_t rows_before, uint32_t r, int gap) {
  return pg_up(rows_before) + r * (uint32_t)gap;
}
// Tiles of all lists, for copies = 1: kPgMostTiles for more than fit, and for a number of rows that
// is none.
__host__ __device__ __forceinline__ uint32_t pg_tiles(int64_t rows, uint32_t lists, int gap) {
  const uint64_t n = (((uint64_t)rows + 31) >> 5) + (uint64_t)lists * (uint32_t)gap;
  return (uint32_t)(rows >= 0 && n < kPgMostTiles ? n : kPgMostTiles);
}
// Whether [p0, p1) are rows of a list, of `rows` of all: offsets that fall, or lie outside the first
// and the last, are the caller's mistake.  A list of such is as one without a row: it has no place.
__host__ __device__ __forceinline__ bool pg_held(int64_t p0, int64_t p1, int64_t rows) {
  return p0 >= 0 && p1 >= p0 && p1 <= rows;
}
// The tiles from a list's first row to the next one's, none of one that is not held: they stop there
// as well.
__host__ __device__ __forceinline__ uint32_t pg_list_tiles(int64_t p0, int64_t p1, int64_t rows) {
  if (!pg_held(p0, p1, rows)) return 0;
  const uint64_t n = (((uint64_t)p1 + 31) >> 5) - (((uint64_t)p0 + 31) >> 5);
  return (uint32_t)(n < kPgMostTiles ? n : kPgMostTiles);
}
// Sums of tiles stop there too.
__host__ __device__ __forceinline__ uint32_t pg_add(uint32_t x, uint32_t y) {
  const uint32_t n = x + y;
  return n < kPgMostTiles ? n : (uint32_t)kPgMostTiles;
}

struct PgCut {
  uint32_t tiles, total;  // of a chunk, of all: 0 where they are too many
  bool fits;
};
// tiles: of the lists, for one copy; parts: chunks taken at once; most: that partials have room for.
__host__ __device__ __forceinline__ PgCut pg_cut(uint32_t copies, uint32_t tiles, uint32_t parts,
                                                 uint32_t most) {
  const uint64_t all = (uint64_t)copies * tiles;
  if (all >= kPgMostTiles) return PgCut{kPgMinTiles, 0, false};
  const uint32_t total = (uint32_t)all;
  uint32_t k = (total + parts - 1u) / parts;
  k = k < kPgMinTiles ? kPgMinTiles : k < kPgMaxTiles ? k : kPgMaxTiles;
  // (more rows than the caller's bound or the pool allow for, as with pages that lists share:
  // longer chunks, so that the partials stay within the workspace)
  if (total > (uint64_t)most * k) k = (total + most - 1u) / most;
  return PgCut{(k + kPgMinTiles - 1u) / kPgMinTiles * kPgMinTiles, total, true};
}

// The chunks that a unit's tiles, one or more, lie in: n from `first` on.  (Of a list that is held
// their end is no later than the total's: below 2^31, and the last of the chunks at most.)
struct PgPieces {
  uint32_t first, n;
};
__host__ __device__ __forceinline__ PgPieces pg_pieces(uint32_t place, uint32_t tiles, uint32_t chunk) {
  const uint32_t first = place / chunk;
  return PgPieces{first, (place + tiles - 1u) / chunk - first + 1u};
}

}  // namespace certkv
