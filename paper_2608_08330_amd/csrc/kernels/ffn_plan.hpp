// Tiles and slices of the feed-forward unit's products (gated_ffn.hip), chosen by a
// model of their times.  Host code only, free of HIP headers.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "token_ops.hpp"

namespace rtcc {
namespace kern {
namespace {

constexpr int kMaxProducts = 3;  // of a launch
constexpr int kFewRows = 16;     // up to these no tiles

enum Epilogue { kPlain, kGated, kGatedGrad };

// Tiles and slices of a launch of products with one contracted length.
enum Tiles { kTiles256, kTiles128, kTiles64, kTiles64Deep };  // deep: four buffers for two
struct Plan {
    Tiles kind;
    int slices, per_slice, steps;
    size_t partial;  // bytes
    double us;       // modelled
};
constexpr int kSizeOf[] = {256, 128, 64, 64};
struct Size {
    int64_t m, n;
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Columns of a result that a tile holds.
inline int cols_of(Tiles kind, Epilogue epi) { return epi == kGated ? kSizeOf[kind] / 2 : kSizeOf[kind]; }
inline int64_t tiles_of(const Size &s, Tiles kind, Epilogue epi) {
    return ceil_div(s.m, kSizeOf[kind]) * ceil_div(s.n, cols_of(kind, epi));
}

// Microseconds of a launch, by which tiles and slices are chosen.  A step takes the
// time of its LDS traffic, some 58 KB loaded a microsecond and CU whatever the tile
// (bf16; 128: 32 KB, 0.5 us, or 0.62 us for a block that has the CU to itself; 256: 64
// KB in 1.4 us, all CUs being busy at a lower clock), so that large tiles win where
// they fill the device and little of their time goes into first loads and results,
// which nothing covers there.  float32 is bound by its products.  Measured against it
// (plain results, kernel times): 16,384 x 384, K 1,536: 128 32 us (modelled 32), 256
// 42 (46), 64 39; 32,768 x 384: 256 44 (46), 128 48 (50); three products of 1,536 x
// 384, K 16,384: 256 in 7 slices 72 + 10 (80), 128 in 4 70 + 7 (84), 64 in 4 113 + 7;
// 500 x 1,024, K 2,816: 64 with four buffers 12 (18), in 4 slices 11 + 5, 64 with two
// 23 (26), 128 33 (35).  It is low for the largest products (16,384 rows, 2,048
// channels, 8,192 hidden: gate and up 982 us, 834 modelled, dX 842, 736, the weights
// 1,208, 1,101) and for 256 with g and u stored over six steps (16,384 x 1,536: 62 to 73,
// 51).
struct Cost {
    int resident;                              // blocks of a CU
    double alone, shared;                      // a step of one block, and of each of several
    double plain, gated, gated_saved, grad;  // first loads and results of a block, or of a CU's together
};
constexpr Cost kCost[2][4] = {
    // float32
    {{1, 0, 0, 0, 0, 0, 0}, {2, 2.0, 2.0, 3, 3, 6, 14}, {5, 0.63, 0.51, 3, 3, 4, 14}, {2, 0.6, 0.51, 2, 2, 3, 8}},
    {{1, 1.4, 1.4, 7, 7, 12, 32}, {2, 0.62, 0.5, 3, 3, 6, 13}, {5, 0.4, 0.24, 3, 3, 4, 6}, {2, 0.26, 0.24, 2, 2, 3, 4}},
};
constexpr double kLaunch = 5.0, kJoin = 5.5, kJoinByte = 0.22e-6;

// large: whether the largest tiles may be taken.
inline Plan plan(int64_t cus, const Size *sizes, int count, bool bf16, int64_t k, int segments, Epilogue epi, bool large, bool saved) {
    const int64_t steps = ceil_div(k, bf16 ? 64 : 32) * segments;
    int64_t values = 0;
    for (int i = 0; i < count; ++i) values += sizes[i].m * sizes[i].n;
    Plan best{};
    double least = 0;
    for (Tiles kind : {kTiles256, kTiles128, kTiles64, kTiles64Deep}) {
        if (kind == kTiles256 && !(bf16 && large)) continue;
        const Cost &c = kCost[bf16][kind];
        int64_t tiles = 0;
        for (int i = 0; i < count; ++i) tiles += tiles_of(sizes[i], kind, epi);
        const double ends = epi == kGated ? (saved ? c.gated_saved : c.gated) : epi == kGatedGrad ? c.grad : c.plain;
        // slices of four steps at least, where the tiles are few
        const int64_t most = epi == kPlain && tiles <= 4 * cus ? std::max<int64_t>(1, std::min<int64_t>(steps / 4, 32)) : 1;
        for (int64_t slices = 1; slices <= most; ++slices) {
            const int64_t each = ceil_div(steps, slices), blocks = ceil_div(tiles * slices, cus);
            auto round = [&](int64_t n) { return n ? double(each) * std::max(c.alone, n * c.shared) + ends : 0.0; };
            double t = kLaunch + double(blocks / c.resident) * round(c.resident) + round(blocks % c.resident);
            if (slices > 1) t += kJoin + double(values) * slices * 4 * kJoinByte;
            if (least == 0 || t < least) {
                least = t;
                best = Plan{kind, int(slices), int(each), int(steps), 0, t};
            }
        }
    }
    best.slices = best.per_slice ? int(ceil_div(best.steps, best.per_slice)) : 1;
    if (best.slices > 1) best.partial = size_t(values) * best.slices * sizeof(float);
    return best;
}

inline Plan plan_gated(const FfnArgs &a, int64_t cus) {
    const Size s{a.rows, a.hidden};
    return plan(cus, &s, 1, a.bf16, a.channels, 1, kGated, true, a.gate);
}
inline Plan plan_down(const FfnArgs &a, int64_t cus) {
    const Size s{a.rows, a.channels};
    return plan(cus, &s, 1, a.bf16, a.hidden, 1, kPlain, true, false);
}
inline Plan plan_dhidden(const FfnArgs &a, int64_t cus) {
    const Size s{a.rows, a.hidden};
    return plan(cus, &s, 1, a.bf16, a.channels, 1, kGatedGrad, true, false);
}
// dX and the weights' gradients: plans of their own launches, or of one for both.
struct Backward {
    bool both;
    Plan x, w;
    size_t partial;  // bytes
};
inline Backward plan_backward(const FfnArgs &a, int64_t cus) {
    Size x{a.rows, a.channels}, s[kMaxProducts];
    int n = 0;
    if (a.dw_gate) s[n++] = {a.hidden, a.channels};
    if (a.dw_up) s[n++] = {a.hidden, a.channels};
    if (a.dw_down) s[n++] = {a.channels, a.hidden};
    const bool dx = a.dx && a.rows > 0;
    Backward b{};
    if (dx) b.x = plan(cus, &x, 1, a.bf16, a.hidden, 2, kPlain, a.w_gate_s == a.w_up_s, false);
    if (n) b.w = plan(cus, s, n, a.bf16, a.rows, 1, kPlain, true, false);
    b.partial = std::max(b.x.partial, b.w.partial);
    if (!dx || !n) return b;
    // One launch: the steps of both over all CUs, or those of a longest block, at the
    // pace of a full CU while there are others' steps beside it and then of its own.
    // 500 rows, 1,024 channels, 2,816 hidden: 26 + 5 us for 14 + 5 + 21; 16,384 rows,
    // 384, 1,536: 112 + 8 for 51 + 72 + 10 (173 where longer blocks came last).
    double least = b.x.us + b.w.us;
    const int64_t wide = a.bf16 ? 64 : 32;
    const int64_t steps_x = 2 * ceil_div(a.hidden, wide), steps_w = ceil_div(a.rows, wide);
    int64_t values_w = 0;
    for (int i = 0; i < n; ++i) values_w += s[i].m * s[i].n;
    const int64_t values_x = x.m * x.n;
    for (Tiles kind : {kTiles128, kTiles64, kTiles64Deep}) {
        const Cost &c = kCost[a.bf16][kind];
        const int64_t tiles_x = tiles_of(x, kind, kPlain);
        int64_t tiles_w = 0;
        for (int i = 0; i < n; ++i) tiles_w += tiles_of(s[i], kind, kPlain);
        for (int64_t sx = 1; sx <= 16 && (sx == 1 || (sx * 4 <= steps_x && tiles_x <= 4 * cus)); sx *= 2)
            for (int64_t sw = 1; sw <= 16 && (sw == 1 || (sw * 4 <= steps_w && tiles_w <= 4 * cus)); sw *= 2) {
                const int64_t each_x = ceil_div(steps_x, sx), each_w = ceil_div(steps_w, sw);
                const int64_t blocks = ceil_div(tiles_x * sx + tiles_w * sw, cus);
                const double all = double(tiles_x * sx * each_x + tiles_w * sw * each_w) / double(cus);
                const double longest = double(std::max(each_x, each_w)), beside = std::max(0.0, all - longest);
                const double together = std::min(longest, beside / (c.resident - 1));
                const double path = together * std::max(c.alone, c.resident * c.shared) + (longest - together) * c.alone;
                double t = kLaunch + double(ceil_div(blocks, c.resident)) * c.plain + std::max(all * c.shared, path);
                if (sx > 1) t += kJoin + double(values_x) * sx * 4 * kJoinByte;
                if (sw > 1) t += kJoin + double(values_w) * sw * 4 * kJoinByte;
                if (t >= least) continue;
                least = t;
                b.both = true;
                b.x = Plan{kind, int(ceil_div(steps_x, each_x)), int(each_x), int(steps_x), 0, t};
                b.w = Plan{kind, int(ceil_div(steps_w, each_w)), int(each_w), int(steps_w), 0, t};
            }
    }
    if (b.both) {
        b.x.partial = b.x.slices > 1 ? size_t(values_x) * b.x.slices * sizeof(float) : 0;
        b.w.partial = b.w.slices > 1 ? size_t(values_w) * b.w.slices * sizeof(float) : 0;
        b.partial = b.x.partial + b.w.partial;  // multiples of 32 bytes
    }
    return b;
}

}  // namespace
}  // namespace kern
}  // namespace rtcc
