// Which tile a product over ragged groups takes, and how its work is cut: rules on sizes alone, plain C++.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace nomad_grouped {

// Tiles of the result, columns x rows (gradients: columns of x x columns of dy).  256 x 256 asks L2 for the fewest bytes an operation (31 a clock
// and compute unit at the matrix cores' peak in bfloat16, of 64; 128 x 128 asks for 62: the gradient of 524,288 rows of 2,048 -> 768
// runs at 1,035 against 890 TFLOP/s), but a unit holds only one, and it wastes more on ragged ends.
enum ProductTile { kProduct256 = 0, kProduct128, kProduct64, kProduct16, kProductFew };   // 256x256, 128x128, 64x128, 16x256, few rows
enum GradientTile { kGradient256 = 0, kGradient128, kGradient64, kGradient16 };           // 256x256, 128x128, 64x64, 128x16

inline int64_t tiles_of(int64_t size, int64_t tile) { return (size + tile - 1) / tile; }

// small: two-byte elements (four-byte ones keep the matrix cores busy sixteen times as long for a byte: 128 x 128 always feeds them)
// w_kc: the weights' k is contiguous
inline ProductTile plan_product(int64_t rows, int64_t groups, int64_t out, bool small, bool w_kc, int64_t units) {
    // tiles of rows there can be: no more than one a row, one a group beyond the whole ones
    const auto row_tiles = [&](int64_t tile) { return std::min(rows, rows / tile + groups); };
    // so few that most units would have none: k is shared instead (2 rows, 768 -> 2,048 in bfloat16: 5.6 us, 15.4 in tiles of 128)
    if (w_kc && rows <= 16 * groups && row_tiles(128) * tiles_of(out, 128) < units) return kProductFew;
    if (out <= 16) return kProduct16;   // (131,072 rows of 256 -> 2 in float32: 44 us, 67 in tiles of 64 columns)
    // narrow tiles read x more often, and are right where wide ones would be empty: 129 columns are three of 64, not two of 128
    // (200,006 rows of 50 -> 129 in float32, elements at the ends one by one on both sides: 118 us, 127 in tiles of 128; 113 now)
    if (out <= 64 || tiles_of(out, 64) * 64 * 9 < tiles_of(out, 128) * 128 * 8) return kProduct64;
    if (!small || out <= 128) return kProduct128;
    // large tiles where they are at least half full and there is one for every compute unit
    if (rows < 128 * groups || tiles_of(rows, 256) * tiles_of(out, 256) < units) return kProduct128;
    return kProduct256;
}

struct GradientPlan {
    GradientTile tile;
    int64_t tiles;       // of a part
    int32_t most;        // rows a part has at most: no more than one compute unit's share of the whole
    int32_t slot_bits;   // places for sums of parts are 2^slot_bits rows apart, no more than the shortest part
    int64_t slots;       // of them; 0 where no group can have two parts
};

inline GradientPlan plan_gradient(int64_t rows, int64_t groups, int64_t in, int64_t out, bool small, int64_t units) {
    GradientPlan plan;
    const int64_t large = tiles_of(in, 256) * tiles_of(out, 256), middle = tiles_of(in, 128) * tiles_of(out, 128), little = tiles_of(in, 64) * tiles_of(out, 64);
    // (131,072 rows, 2 x 256 in float32: 58 us, 100 in tiles of 64 x 64)
    if (out <= 16 && in > 64) { plan.tile = kGradient16; plan.tiles = tiles_of(in, 128) * tiles_of(out, 16); }
    else if (small && in > 128 && out > 128 && large * groups >= units / 2) { plan.tile = kGradient256; plan.tiles = large; }
    else if (little * 16 < middle * 48) { plan.tile = kGradient64; plan.tiles = little; }   // a quarter less to compute, or more (40,022 rows, 50 x 129 in float32, elements at the ends one by one on both sides: 42 us, 68 in tiles of 128; 34 now)
    else { plan.tile = kGradient128; plan.tiles = middle; }
    // A quarter of a workgroup's share of the whole, so that they end together (groups of 8,192 rows, 2,048 x 768 in bfloat16: 2.1 ms, 2.5
    // with whole shares).  But a part's sums are written and read once more: as many bytes as reading some rows, and no part has fewer
    // than eight times those (256 x 256 in bfloat16: 4,096; groups of 800 rows, 512 x 768: 0.29 ms, 0.41 with quarters of a
    // share) unless the share itself is less; nor fewer than 256, four stages of the products.
    const int64_t a = plan.tile == kGradient256 ? 256 : plan.tile == kGradient64 ? 64 : 128, b = plan.tile == kGradient16 ? 16 : a;
    const int64_t share = rows * plan.tiles / (units * (plan.tile == kGradient256 ? 1 : 2)), least = 8 * (a * b * 8) / ((a + b) * (small ? 2 : 4));
    plan.most = (int32_t)std::min<int64_t>(std::max<int64_t>({256, share / 4, std::min(share, least)}), (int64_t)1 << 30);
    plan.slot_bits = 0;
    while ((int64_t)2 << plan.slot_bits <= plan.most / 2) ++plan.slot_bits;
    plan.slots = rows > plan.most ? (rows >> plan.slot_bits) + 1 : 0;
    return plan;
}

}  // namespace nomad_grouped
