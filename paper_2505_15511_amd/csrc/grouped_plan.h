// Which tile a product over ragged groups takes, and how its work is cut: rules on sizes alone, plain C++.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace nomad_grouped {

// Tiles of the result, columns x rows (gradients: columns of x x columns of dy).  256 x 256 needs the fewest bytes from L2 an operation (31 a clock and
// compute unit at the matrix cores' peak, of 64; 128 x 128 needs 62, and reaches 890 TFLOP/s where the large one reaches
// 990 in bfloat16), but a unit holds only one, and it wastes more on ragged ends.
enum ProductTile { kProduct256 = 0, kProduct128, kProduct64, kProduct16 };   // 256x256, 128x128, 64x128, 16x256
enum GradientTile { kGradient256 = 0, kGradient128, kGradient16 };           // 256x256, 128x128, 128x16

inline int64_t tiles_of(int64_t size, int64_t tile) { return (size + tile - 1) / tile; }

// small: two-byte elements (four-byte ones keep the matrix cores busy sixteen times as long for a byte: 128 x 128 always feeds them)
inline ProductTile plan_product(int64_t rows, int64_t groups, int64_t in, int64_t out, bool small, int64_t units) {
    (void)in;
    if (out <= 16) return kProduct16;
    if (out <= 64) return kProduct64;
    if (!small || out <= 128) return kProduct128;
    // large tiles where they are at least half full and there is one for every compute unit
    if (rows < 128 * groups || tiles_of(rows, 256) * tiles_of(out, 256) < units) return kProduct128;
    return kProduct256;
}

struct GradientPlan {
    GradientTile tile;
    int64_t tiles;   // of a part
    int32_t most;    // rows a part has at most: no more than one compute unit's share of the whole
    int64_t slots;   // places for sums of parts; 0 where no group can have two
};

inline GradientPlan plan_gradient(int64_t rows, int64_t groups, int64_t in, int64_t out, bool small, int64_t units) {
    GradientPlan plan;
    const int64_t large = tiles_of(in, 256) * tiles_of(out, 256);
    if (out <= 16) plan.tile = kGradient16;
    else if (!small || in <= 128 || out <= 128 || large * std::max<int64_t>(groups, 1) < units / 2) plan.tile = kGradient128;
    else plan.tile = kGradient256;
    plan.tiles = plan.tile == kGradient256 ? large : tiles_of(in, 128) * tiles_of(out, plan.tile == kGradient16 ? 16 : 128);
    // a part's sums cost as much as some hundred rows: no shorter than 256
    const int64_t share = rows * plan.tiles / units;
    plan.most = (int32_t)std::min<int64_t>(std::max<int64_t>(256, share), (int64_t)1 << 30);
    plan.slots = rows > plan.most ? rows / (plan.most / 2) + 1 : 0;
    return plan;
}

}  // namespace nomad_grouped
