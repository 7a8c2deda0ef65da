// The tile of a product of 8-bit integers (linear_i8.h), chosen on the host.  No HIP in it: linear_i8_tiles_driver.cpp asks it too.
#pragma once
#include <math.h>

namespace thia {

// Which tile: the one with the least base + K tiles * (per_k * rounds + more_k * (r - 1)) + per_tile * r, in us, where r is the number of tiles
// per CU, at least 1, and `rounds` that number rounded up.  The constants are a least-squares fit (relative errors) to what the tiles took on
// 240 shapes of 1 to 16 384 rows, 128 to 12 544 columns and 64 to 8 192 channels; over these the rule is 1.4 % from the best tile in the geometric
// mean, and 29 % at worst.  Measured in us (bf16 results, back to back in a captured graph), rows x columns x channels:
//                        16x16  32x32  32x64  64x64  96x64  128x64  128x128  192x256  256x256
//   1 x 4096 x 4096        3.3    4.3    5.1    6.6
//   130 x 4096 x 512       7.1    4.4    5.3    7.2
//   700 x 256 x 2048       9.4    6.0    4.4    5.0    5.3     6.5      6.8      8.4
//   700 x 12544 x 1024             34     28     21     25      30
//   1200 x 12544 x 1024            69     45     39     27      31       45
//   2000 x 12544 x 1024           112     63     60     57      39       46
//   4000 x 1024 x 1024             21     14     13     16      16       10       13       16
//   9600 x 1024 x 1024                    32     31     42      43       27       17       18
//   4000 x 4096 x 4096                                                   97       78       60
//   9600 x 12544 x 1024                                                 159      106      114
// It does not know whether rows take 16-byte accesses: with odd channels and a residual the epilogue of the larger tiles outweighs the rest (see finish_rows).
struct Tile { int rows, chans; double base, per_k, per_tile, more_k; };
constexpr Tile kTiles[] = {{16, 16, 2.67, 0.065, 0.120, 0.038},  {32, 32, 2.61, 0.060, 0.515, 0.018},   {32, 64, 2.77, 0.088, 0.513, 0.042},
                           {64, 64, 2.61, 0.139, 1.366, 0.061},  {96, 64, 0.58, 0.224, 4.041, 0.0},     {128, 64, 1.53, 0.271, 4.688, 0.056},
                           {128, 128, 0.41, 0.448, 6.220, 0.139}, {192, 256, 0.0, 0.824, 8.133, 0.739}, {256, 256, 0.0, 1.051, 9.378, 0.982}};

inline int choose_tile(int rows, int n, int pitch) {
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
        const Tile& t = kTiles[i];
        if (t.chans == 256 && pitch < 256) continue;   // two K tiles are under way there
        const double tiles = (double)((rows + (long long)t.rows - 1) / t.rows) * ((n + t.chans - 1) / t.chans);
        const double r = tiles > 256 ? tiles / 256 : 1.0;
        double k_tiles = pitch / 128;
        if (t.rows == 16) k_tiles *= 0.5 + 0.03125 * (rows < 16 ? rows : 16);   // rows that do not exist are not fetched
        const double us = t.base + k_tiles * (t.per_k * ceil(tiles / 256) + t.more_k * (r - 1)) + t.per_tile * r;
        if (i == 0 || us < least) { best = i; least = us; }
    }
    return best;
}

}  // namespace thia
