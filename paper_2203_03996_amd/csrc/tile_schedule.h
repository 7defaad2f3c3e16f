// How products are cut into tiles, when K-tiles are copied into LDS and what is waited for before they are read.  Plain C++: the tests
// compile it for the host.
#pragma once

namespace dcnn {

// Tiles of `per` rows that cover `rows` (to 2^31 - 1: nothing here may pass it on the way).
constexpr int tiles_of(int rows, int per) { return rows / per + (rows % per != 0); }
// Row `row` of the tile that begins at row t0 is one of the `rows` there are.
constexpr bool in_rows(int t0, int row, int rows) { return row < rows - t0; }

// A workgroup takes tiles one behind the other, each of `kts` K-tiles; K-tile kt of a tile lies in buffer kt % nb.  Copies are issued in the
// order of use and arrive in the order of issue: before the first tile those of its K-tiles 0 .. nb - 1 (as many as there are), then one
// behind every K-tile, into the buffer that this K-tile leaves, while there are tiles left to be copied (`more`).

// The K-tile that is copied into the buffer that K-tile kt leaves: of this tile, or (turns_to_next) of the one behind it.
constexpr int copied_behind(int kt, int kts, int nb) { return kt + nb < kts ? kt + nb : kt % nb; }
// ... is the first of the next tile's.
constexpr bool turns_to_next(int kt, int kts, int nb) { return kt + nb == kts || (kts < nb && kt == 0); }
// Copied K-tiles that may still be on their way in a workgroup's first tile when K-tile kt + 1 has to be there (in later tiles: from
// kt + 1 = nb on, those before have been waited for): the ones issued behind it.  A tile of fewer than nb K-tiles has fewer on their way.
constexpr int may_be_in_flight(int kt, int kts, int nb, bool more) {
    if (nb == 2) return 0;
    const int behind = more && kts >= nb ? nb - 2 : kts - 2 - kt;          // (a tile of fewer than nb: the first wait is at kt = 0, later ones need less)
    return behind > 0 ? behind : 0;
}

}  // namespace dcnn
