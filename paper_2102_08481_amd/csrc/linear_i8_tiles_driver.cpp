// The tile that each product of 8-bit integers takes (no GPU): reads "rows columns channels" lines, prints "rows x channels" of the tile.
// Built and run by tests/test_i8_tiles.py, not part of libthia.so.
#include <cstdio>

#include "linear_i8_tiles.h"

int main() {
    int rows, k, n;
    while (std::scanf("%d %d %d", &rows, &k, &n) == 3) {
        const thia::Tile& t = thia::kTiles[thia::choose_tile(rows, n, (k + 127) / 128 * 128)];
        std::printf("%dx%d\n", t.rows, t.chans);
    }
}
