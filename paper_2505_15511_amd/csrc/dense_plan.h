// How a dense product is cut: rules on sizes alone, plain C++.
#pragma once
#include <stdint.h>

#include <algorithm>

#include "grouped_plan.h"

namespace nomad_dense {

using nomad_grouped::tiles_of;

// Tiles of the result, its contiguous columns x its rows
enum Tile { k256 = 0, k128, k64, k16, kFew };   // 256x256, 128x128, 64x128, 16x256; few rows: 16 columns x up to 64 rows

struct Plan {
    Tile tile;
    int64_t parts;     // the sum over k is cut into
    int64_t length;    // k of a part, a multiple of a stage's
    int64_t units;     // tiles times parts
};

constexpr int64_t kFewRows = 64, kMostParts = 64;

// Whether tiles of 256 fill the units, by themselves or with a sum cut into parts of at least 1,024 (65,536 rows, weights' gradient of 2,048 x 768
// in bfloat16: 250 us in ten parts of 24 such tiles, 266 in five of 96 tiles of 128; with parts of 256 already, 130 rows of 4,096 -> 4,096
// take 28 us, 21 in tiles of 128)
// (The columns that the last tile leaves empty are not looked at: 65,536 rows of 512 -> 328 and 576 take 54 and 63 us, 40 and 59 in tiles of 128.)
inline bool large(int64_t rows, int64_t columns, int64_t k, int64_t units) {
    const int64_t tiles = tiles_of(rows, 256) * tiles_of(columns, 256);
    return tiles >= units || (rows > 128 && columns > 128 && units / tiles * 1024 <= k && units / tiles * tiles * 8 >= units * 7);
}

// rows x columns of the result, k of the sum; small: two-byte elements; few: rows are read as k runs on either side; whole: 16-byte chunks
// on either side and of the result
inline Plan plan(int64_t rows, int64_t columns, int64_t k, bool small, bool few, bool whole, int64_t units) {
    Plan p;
    const int64_t stage = small ? 64 : 32;
    int64_t a, b, at_once;
    if (few && rows <= kFewRows) { p.tile = kFew; a = 16; b = kFewRows; at_once = 1; }
    else if (columns <= 16) { p.tile = k16; a = 16; b = 256; at_once = 2; }
    // (tiles of 64 columns and of 128, us: 65,536 rows of 512 in float32 to 136, 192, 320 and 448 columns 116, 118, 187, 268 and 144, 142, 210, 278; to 328 and 456, where
    // those of 128 leave less of themselves empty, 225, 296 and 212, 276; 2,000 rows of 1,024 in bfloat16 to 192 14.6 and 16.0, 65,536 rows of 512 28.6 and 27.8)
    else if (columns <= 64 || tiles_of(columns, 64) * 64 * 9 < tiles_of(columns, 128) * 128 * 8) { p.tile = k64; a = 64; b = 128; at_once = 2; }
    else if (small && whole && large(rows, columns, k, units)) { p.tile = k256; a = 256; b = 256; at_once = 1; }
    else { p.tile = k128; a = 128; b = 128; at_once = 2; }
    const int64_t tiles = tiles_of(columns, a) * tiles_of(rows, b), stages = tiles_of(k, stage);
    // Where tiles leave units without work, the sum is cut, to no less than four stages (500 rows of 8,192 -> 768 in bfloat16: 22 us, 25 with sixteen at
    // least), for few rows to no less than sixteen, two rounds of the loads that a wavefront has on their way (24 rows of 8,192 -> 4,096 in
    // float16: 24.5 us in one part, 27.4 in two; one row of 768 -> 2,048: 9 us, 17 in three parts, whose sums are a second launch); and to no more than
    // 64 parts, whose sums are written and read once more (65,536 rows, weights' gradient of 256 x 256: 31 us, 37 in 128 parts)
    p.parts = std::max<int64_t>(1, std::min({units * at_once / tiles, stages / (p.tile == kFew ? 16 : 4), kMostParts}));
    const int64_t per = std::max<int64_t>(1, tiles_of(stages, p.parts));
    p.length = per * stage;
    p.parts = std::max<int64_t>(1, tiles_of(stages, per));
    p.units = tiles * p.parts;
    return p;
}

// Rows of a part of dz = dy act'(z), whose sums over rows meet afterwards: parts for all units, with at least 64 rows, and no more than 512 of them. (dz, db and a dW of 8
// columns, 65,536 rows of 2,048 in bfloat16: 230 us, with 128 parts at most 481, with 2,048 236; a million rows of 128 385, 627 and 401. 2, 4, 16 or 32 times the units in place of
// 8 change nothing, 227 to 229 us.)
struct SlopePlan { int64_t parts, length; };
inline SlopePlan plan_slope(int64_t rows, int64_t columns, int64_t units) {
    const int64_t strips = tiles_of(columns, 2048);   // (as many columns as a workgroup takes side by side, or fewer)
    const int64_t parts = std::max<int64_t>(1, std::min({rows / 64, (int64_t)512, std::max<int64_t>(1, 8 * units / strips)}));
    SlopePlan p;
    p.length = std::max<int64_t>(1, tiles_of(rows, parts));
    p.parts = std::max<int64_t>(1, tiles_of(rows, p.length));
    return p;
}

}  // namespace nomad_dense
