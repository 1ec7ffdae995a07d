// What kernel takes which product of the gated feed-forward block, and how the tiles of a launch are divided.  Index arithmetic alone, without any HIP
// header, so that a host program can walk through it.
#pragma once

#include <algorithm>

#include "hdt.h"

namespace hdt_ffn {

template <int WM_, int WN_, int MB_, int NB_, int BK_, int STAGES_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, NW = WM * WN, THREADS = NW * 64;
    static constexpr int BM = WM * MB * 32, BN = WN * NB * 32, BK = BK_, STEPS = BK / 16, STAGES = STAGES_;
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2, STAGE = A_BYTES + B_BYTES, LDS = STAGES * STAGE;
    static constexpr int LOADS = (BM + BN) * BK / 8 / 64 / NW;  // direct loads of a stage, for each wave
};
using Large = Shape<2, 4, 4, 2, 32, 4>;  // 256 x 256, a workgroup a compute unit
using Small = Shape<2, 2, 2, 2, 64, 2>;  // 128 x 128, two

// Products that one launch makes in tiles, and how (TileArgs has the meanings).
struct Plan {
    int shape;  // 0 Large, 1 Small
    unsigned direct, tiles, piece_items, sharers;
    int pieces, per, rest;
    size_t parts_bytes;
};
struct Dims {
    int m, n;  // n: columns of the tile's operand (of both weights, for GATE)
};
inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// The rule is a sum of clocks: a walk along k, what stands around it, and the parts of tiles that are cut.  slots: workgroups the chip holds; step,
// around: clocks of 64 of k with every unit full, and of what stands around a tile's walk.  As measured (us of forward and backward, kernels, Large |
// Small): 32768 x 768 x 2048 1184 | 1413, 8192 x 1024 x 4096 741 | 799, 1999 x 1000 x 2504 240 | 200, 512 x 768 x 2048 137 | 101.  A unit with one
// Small workgroup is no quicker a step than with two.
template <typename S>
void consider(const Dims *of, int products, int k, int ranges, bool divisible, int shape, unsigned slots, double step, double around, Plan *best, double *best_cost)
{
    int64_t tiles = 0;
    for (int i = 0; i < products; i++) tiles += (int64_t)ceil_div(of[i].m, S::BM) * ceil_div(of[i].n, S::BN);
    const int k_tiles = ranges * ceil_div(k, S::BK);
    step *= S::BK / 64.;
    auto offer = [&](const Plan &plan, double cost) {
        if (*best_cost >= 0 && cost >= *best_cost) return;
        *best_cost = cost;
        *best = plan;
    };
    const double rounds = (double)((tiles + slots - 1) / slots);
    offer({shape, (unsigned)tiles, (unsigned)tiles, 0, 0, 0, 0, 0, 0}, rounds * (k_tiles * step + around));
    const int64_t direct = tiles / slots * slots, cut = tiles - direct;
    if (!divisible || cut == 0 || k_tiles == 0) return;
    const int least = std::min(256 / S::BK, k_tiles);  // (shorter walks are their beginning and end)
    const double before = (double)(direct / slots) * (k_tiles * step + around);
    auto cut_into = [&](int pieces, int per, int rest) {
        const int64_t sharing = rest ? ceil_div(cut * rest, per) : 0, items = cut * pieces + sharing;
        const unsigned piece_items = (unsigned)(cut * pieces + 7) / 8 * 8, sharers = (unsigned)(sharing + 7) / 8 * 8;
        // parts are written and read at about 3000 bytes a clock; and a launch
        const size_t parts = (size_t)(cut * pieces + (rest ? sharers + cut : 0)) * S::BM * S::BN * sizeof(float);
        const double tiles_of_one = rest ? per / (double)rest + 1 : 1;
        offer({shape, (unsigned)direct, (unsigned)tiles, piece_items, sharers, pieces, per, rest, parts},
              before + (double)ceil_div(items, slots) * (per * step + tiles_of_one * around) + parts * 2. / 3000 + 8000);
    };
    // The chip's share each, the rest divided anew; or equal pieces, the last a little shorter.  Either way a tile that is cut has two parts or more, in different
    // workgroups (there are fewer such tiles than slots, so a share is at most a tile: one piece or more, and where it is not all of the tile a rest).
    const int share = std::max(ceil_div(cut * k_tiles, slots), least), pieces = k_tiles / share, rest = k_tiles - pieces * share;
    if (rest) cut_into(pieces, share, rest);
    for (int n = 2; n <= 32; n++) {
        const int per = ceil_div(k_tiles, n);
        if (per >= least && ceil_div(k_tiles, per) == n) cut_into(n, per, 0);
    }
}
inline Plan plan_of(const Dims *of, int products, int k, int ranges, bool divisible)
{
    Plan best = {};
    double cost = -1;
    consider<Large>(of, products, k, ranges, divisible, 0, 256, 4000, 9000, &best, &cost);
    consider<Small>(of, products, k, ranges, divisible, 1, 512, 2800, 7000, &best, &cost);
    return best;
}

// How many rows are few depends on the weights, which each group of at most 64 rows reads anew (us, forward, this way | in tiles: 1024 x 2816 64 rows 11.5 | 38,
// 128 15.3 | 31, 192 21 | 34; 768 x 2048 128 11.6 | 20, 192 15.6 | 22; 4096 x 1024 192 30 | 67; 2048 x 4096 128 32 | 45, 192 49 | 48; 2048 x 8192 64 33 | 51,
// 128 55 | 52; 4096 x 11008 64 89 | 107, 128 146 | 109).
inline bool few_rows(int64_t rows, int width, int inner)
{
    const int64_t weights = (int64_t)width * inner;
    return rows <= 64 || (rows <= 128 && weights <= 1 << 24) || (rows <= 192 && weights <= 1 << 22);
}

// Tiles of 64 x 64; where those do not fill the chip four groups of a workgroup divide k, and where they do not give each compute unit one,
// tiles of 32 x 32, eight of whose waves divide k (512 x 384 x 1000, forward and backward, us, when a load was one value: one group 752, four 205,
// all three 160)
enum class PlainForm { kSmallDivided, kDivided, kWhole };
inline PlainForm plain_form(int64_t tiles) { return tiles <= 256 ? PlainForm::kSmallDivided : tiles <= 512 ? PlainForm::kDivided : PlainForm::kWhole; }
inline int64_t plain_tiles(Dims d) { return ((int64_t)d.m + 63) / 64 * (((int64_t)d.n + 63) / 64); }

inline size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Sizes {
    int64_t rows;
    int width, inner;
    hdt_dtype_t dt;
    size_t hidden_bytes() const { return padded((size_t)rows * inner * (dt == HDT_BF16 ? 2 : 4)); }
    bool tiled() const { return dt == HDT_BF16; }
    // whether rows begin at multiples of 16 bytes, as direct loads need it
    bool even() const { return width % 8 == 0 && inner % 8 == 0; }
    bool few() const { return tiled() && few_rows(rows, width, inner); }  // (the forward's products)
    Plan plan_gate() const
    {
        const Dims d = {(int)rows, 2 * inner};
        return plan_of(&d, 1, width, 1, false);
    }
    Plan plan_down() const
    {
        const Dims d = {(int)rows, width};
        return plan_of(&d, 1, inner, 1, true);
    }
    Plan plan_dgate() const
    {
        const Dims d = {(int)rows, inner};
        return plan_of(&d, 1, width, 1, false);
    }
    Plan plan_dx() const
    {
        const Dims d = {(int)rows, width};
        return plan_of(&d, 1, inner, 2, true);
    }
    Plan plan_weights() const
    {
        const Dims d[] = {{inner, width}, {inner, width}, {width, inner}};
        return plan_of(d, 3, (int)rows, 1, true);
    }
    size_t fwd_bytes(bool train) const { return (train ? 0 : hidden_bytes()) + (tiled() && !few() ? plan_down().parts_bytes : 0); }
    size_t bwd_bytes() const { return 2 * hidden_bytes() + (tiled() ? std::max(plan_dx().parts_bytes, plan_weights().parts_bytes) : 0); }
};

}  // namespace hdt_ffn
