// Which tiles a weight gradient (ll_act_wgrad) is cut into, and over how many runs
// of tokens.  Plain C++ without HIP, so that it can be compiled and checked by itself.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace lossy {

constexpr int kStepT = 32;  // tokens of a step

// The tiles of all workers in order; the first `whole` are summed by a workgroup
// each, the other `rest` by `runs` workgroups over run_t tokens each, whose
// fp32 sums (tile by tile, [rest][runs][edge][edge]) a second launch joins.
struct WgradPlan {
    int edge;    // of the square tiles
    bool light;  // light workgroups
    int64_t tiles_o, tiles_h, whole, rest;
    int runs;
    int64_t run_t;
    float* part;
};

// Microseconds of a plan, from measurements on layers of 256 to 6000 columns and 2 to
// 8192 tokens: a launch with its first loads and last stores, a step of 32 tokens
// where few compute units work, where each has a tile and where each has as many
// as fit, and what a further round of tiles costs besides its steps.  Sums kept
// apart cost 3 and 0.27 a megabyte.  bf16 dy and gradients (256 x 256 / 128 x 128 /
// light): 32 tokens, 4096 x 4096 13.0 / 16.6 / 10.7; 256 tokens 17.2 / 21.8 / 18.5; 4
// workers' 128 tokens 48.6 / 58.6 / 40.7, 512 tokens 88.3 / 106.9 / 88.7; 512 tokens, 2048
// x 2048 18.8 / 12.1 / 12.9; 3 workers' 10 tokens, 3936 x 5312 40 / 48 / 27.  Runs: 512
// tokens, 2048 x 2048 by 128 x 128 tiles one 12.1, two 33.5; 8192 tokens by 256 x 256 four
// 77.4, one 156.4; fp32, 2048 tokens by 128 x 128 two 62.3, one 63.4.  16384 tokens of
// 512 x 1024 (32 tiles of 128 x 128) into fp32, events between the calls: 4 runs 49, 8
// 36, 12 40, 16 39, 20 44, 24 45, 32 48; the model takes 16.
constexpr int64_t kCus = 256;

struct TileCost {
    int edge, places;  // workgroups that fit a compute unit
    bool light;
    double launch, few, one, all, round;
};
constexpr TileCost kCost[2][3] = {  // [bf16]
    {{256, 1, false, 11.0, 1.69, 2.30, 2.30, 9.0}, {128, 2, false, 7.0, 0.83, 0.83, 1.40, 4.5}},
    {{256, 1, false, 11.0, 0.57, 0.80, 0.80, 9.0},
     {128, 2, false, 6.7, 0.35, 0.40, 0.55, 4.5},
     {128, 4, true, 5.9, 0.40, 0.44, 1.11, 4.3}},
};

inline double tiles_us(const TileCost& c, int64_t blocks, int64_t steps) {
    const int64_t places = c.places * kCus, full = blocks / places, rest = blocks - full * places;
    const double last = rest == 0      ? 0.0
                        : rest <= kCus ? c.few + (c.one - c.few) * rest / kCus
                                       : c.one + (c.all - c.one) * (rest - kCus) / (places - kCus);
    // light workgroups end one by one
    const double rounds = c.light ? (double)blocks / places : full + (rest > 0) - 1;
    return steps * (full * c.all + last) + c.round * rounds;
}

inline void wgrad_plan(int64_t n, int64_t t, int64_t o, int64_t h, bool bf16, WgradPlan* g) {
    const int64_t steps = (t + kStepT - 1) / kStepT;
    double best = 0.0;
    for (const TileCost& cost : kCost[bf16]) {
        if (cost.edge == 0) break;
        const int edge = cost.edge;
        const int64_t tiles_o = (o + edge - 1) / edge, tiles_h = (h + edge - 1) / edge;
        const int64_t tiles = n * tiles_o * tiles_h;
        const int64_t places = cost.places * kCus;
        for (int64_t runs = 1; runs <= 64 && (runs == 1 || runs * 2 <= steps); ++runs) {
            if (runs > 1 && cost.light) break;
            const int64_t whole = runs == 1 ? tiles : tiles / places * places;
            const int64_t rest = tiles - whole;
            if (runs > 1 && (rest == 0 || rest * runs > 4 * kCus)) break;
            int64_t each = (steps + runs - 1) / runs;
            if (each < 1) each = 1;
            double us = cost.launch + (whole > 0 ? tiles_us(cost, whole, steps) : 0.0);
            if (runs > 1)
                us += tiles_us(cost, rest * runs, each) + 3.0 +
                      0.27e-6 * rest * runs * edge * edge * 4 + (whole > 0 ? cost.round : 0.0);
            if (g->edge && us >= best) continue;
            best = us;
            g->edge = edge;
            g->light = cost.light;
            g->tiles_o = tiles_o;
            g->tiles_h = tiles_h;
            g->whole = whole;
            g->rest = rest;
            // as many runs as have tokens
            g->runs = runs == 1 ? 1 : (int)((steps + each - 1) / each);
            g->run_t = each * kStepT;
        }
    }
}

// Bytes of the partial sums.
inline size_t wgrad_part_bytes(const WgradPlan& g) {
    return g.runs > 1 ? (size_t)g.rest * g.runs * g.edge * g.edge * 4 : 0;
}

}  // namespace lossy
