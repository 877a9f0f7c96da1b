// Host side of the layer operators' products: the tile of a workgroup and the
// parts that a long sum is cut into.  Plain C++ (no HIP), so that CPU tests
// can build it on its own.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <limits>

namespace layer_plan {

constexpr int kCus = 256;
constexpr int64_t kMaxBlocks = 0x3fffff;   // workgroups of a launch: fewer than 2^32 threads

inline int64_t tiles(int64_t size, int64_t tile) { return (size + tile - 1) / tile; }

// How a product is cut up: the tile of a workgroup, and the parts that the
// contracted axis is split into where there would be too few workgroups.
struct TileCost {
    int bm, bn;
    int resident;                // workgroups of a CU at a time
    float alone_us, full_us;     // a step of the contracted axis, with few workgroups and with all CUs full
    float fixed_us;              // what a workgroup takes besides
};

struct Plan {
    int tile = 0, split = 1;
    int64_t tiles_m = 0, tiles_n = 0, blocks = 0;
    size_t workspace = 0;
};

// The cheapest of the tiles and splits by the time at which the last CU ends,
// with what joining the parts costs: a launch, and every part written and
// read.  The times were measured on MI355X over sizes from one token to
// 65,536 and widths of 96 to 8,192.
inline Plan plan_product(const TileCost *tile, int count, int64_t n, int64_t m, int64_t cols, int64_t steps) {
    Plan best;
    float best_us = 0.0f;
    for (int c = 0; c < count; ++c) {
        const TileCost &t = tile[c];
        const int64_t tm = tiles(m, t.bm), tn = tiles(cols, t.bn), places = kCus * t.resident;
        // The last one fills the chip just once.
        const int once = (int)std::min<int64_t>(64, places / std::max<int64_t>(1, n * tm * tn));
        for (const int split : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, once}) {
            if (split < 1 || (split > steps && split > 1)) continue;
            const int64_t blocks = n * tm * tn * split;
            const float fill = std::min(1.0f, (float)blocks / (float)places);
            const float step = t.alone_us + (t.full_us - t.alone_us) * fill;
            float us = (float)tiles(blocks, places) * (t.fixed_us + (float)tiles(steps, split) * step);
            if (split > 1) us += 2.5f + (float)(split + 1) * (float)n * (float)m * (float)cols * 4.0f / 3.5e6f;
            // More workgroups than a launch can have: only if nothing else is left.
            if (blocks > kMaxBlocks) us = std::numeric_limits<float>::infinity();
            if (best.blocks && us >= best_us) continue;
            best_us = us;
            best = Plan{c, split, tm, tn, blocks, split > 1 ? (size_t)split * n * m * cols * 4 : 0};
        }
    }
    return best;
}

inline Plan plan_linear(int32_t n, int64_t tokens, int64_t width, int64_t channels) {
    static const TileCost tile[] = {{256, 256, 1, 1.35f, 2.0f, 4.5f},
                                    {64, 128, 3, 0.4f, 1.0f, 4.0f},
                                    {16, 128, 4, 0.35f, 0.9f, 3.0f}};
    return plan_product(tile, 3, n, tokens, channels, tiles(width, 128));
}

// The gradients' tiles: the first as large as two of its steps fit in LDS.
inline Plan plan_grad(int32_t type, int64_t n, int64_t m, int64_t cols, int64_t r) {
    static const TileCost tile[3][2] = {{{128, 128, 1, 1.65f, 1.95f, 4.5f}, {64, 128, 2, 1.35f, 2.3f, 4.0f}},
                                        {{256, 256, 1, 1.65f, 2.0f, 5.0f}, {64, 128, 3, 0.75f, 1.45f, 3.5f}},
                                        {{128, 256, 1, 1.8f, 2.3f, 4.5f}, {64, 128, 2, 1.25f, 1.8f, 3.5f}}};
    return plan_product(tile[type], 2, n, m, cols, tiles(r, 64));
}

}  // namespace layer_plan
