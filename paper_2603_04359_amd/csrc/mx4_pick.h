// The form and the tile shape that a product of MXFP4 codes takes, from its
// sizes alone: host code, without the device.
#pragma once

#include <cmath>
#include <cstdint>

namespace catk {

struct Mx4Sizes {
    int n, m, groups, d_in, d_out;         // rows of x, rows of y, experts (1: dense)
    bool by_expert, gathered;              // with offsets, with row ids
};

enum class Mx4Form { split, line, tile };
struct Mx4Pick {
    Mx4Form form;
    int shape;                             // index into the form's list
    bool whole;                            // rows need no general arithmetic
};

// Short rows: a wave for each chunk of 128 elements.
constexpr int kSpWaves = 4;                // at most
constexpr int kSpRow = 512;                // elements that a row has less of
static_assert(kSpRow == 128 * kSpWaves, "a wave for each chunk, none without");

// Accumulators whose partial sums are added at a time: one per wave.
constexpr int mx4_round(int a, int b, int w) { return a * b < w ? a * b : w; }
// LDS of a wave: its copies, later its partial sums of a round.
constexpr int mx4_wave_bytes(int a, int b, int w, int ring) {
    return ring > mx4_round(a, b, w) * 1024 ? ring : mx4_round(a, b, w) * 1024;
}
constexpr int sp_wave_bytes(int a, int b, bool aligned) {
    return mx4_wave_bytes(a, b, kSpWaves, (a + b) * 1024 + (a + b + 3) / 4 * 256 * (aligned ? 1 : 2));
}

// Rows of 512 elements and more, chunks of 256.
constexpr int ln_scale_bytes(int a, int b) { return (a + b + 1) / 2 * 1024; }
constexpr int ln_stage_bytes(int a, int b) { return 2 * (a + b) * 1024; }
constexpr int ln_wave_bytes(int a, int b, int d, int w) {      // as many scale buffers as chunks
    return mx4_wave_bytes(a, b, w, d * (ln_stage_bytes(a, b) + ln_scale_bytes(a, b)));
}

// Tile shapes of the split kernel: rows / 16, outputs / 16.
#define CAT_SPLIT_TILES(V) V(0, 1, 1) V(1, 1, 2) V(2, 1, 4) V(3, 2, 4) V(4, 4, 4)
// Of the line kernel: rows / 16, outputs / 16, ring chunks, waves.
#define CAT_LINE_TILES(V) \
    V(0, 1, 1, 2, 8) V(1, 1, 2, 2, 4) V(2, 1, 4, 1, 4) V(3, 2, 2, 2, 4) V(4, 2, 4, 1, 4) V(5, 3, 4, 1, 4) \
    V(6, 4, 4, 1, 4)
struct SmallTile {
    int a, b, d, w;
};
#define CAT_SHAPE(id, A, B) {A, B, 1, kSpWaves},
static constexpr SmallTile kSpTiles[] = {CAT_SPLIT_TILES(CAT_SHAPE)};
#undef CAT_SHAPE
#define CAT_SHAPE(id, A, B, D, W) {A, B, D, W},
static constexpr SmallTile kLnTiles[] = {CAT_LINE_TILES(CAT_SHAPE)};
#undef CAT_SHAPE
// Of the tile kernel: rows, outputs.
struct LargeTile {
    int bm, bn;
};
static constexpr LargeTile kTlTiles[] = {{128, 128}, {128, 256}, {256, 256}};

// Row tiles to expect.  Where rows go is known on the device only: their
// counts are taken as exponentially distributed over the experts that have
// any (a router prefers some), which gives 1 / (1 - exp(-bm / mean)) tiles each.
inline double row_tiles(const Mx4Sizes& a, int bm) {
    if (!a.by_expert) return static_cast<double>((a.m + bm - 1) / bm);
    const double used = a.groups * (1.0 - std::exp(-static_cast<double>(a.m) / a.groups));
    return used / (1.0 - std::exp(-bm * used / a.m));
}

// Estimated nanoseconds.  Small tiles: the workgroups of a CU that fit its LDS
// and waves run together, so a CU's tiles cost their rounds at the latency of
// the chunks of a wave (580 ns each, 360 with two in flight) or their sum at
// the rate of its copies (13.9 ns each) and of the sums, whichever is longer.
// Large tiles: rounds, pairs and a fixed part; 128 x 128 outputs run two a CU,
// a pair of both in 1.2 us where one alone takes 0.64.  Over 800 random shapes
// (1 to 4096 rows, dense and by up to 128 experts, 1024 to 14336 inputs, 128 to
// 16384 outputs) the shape with the least estimate took 2.7% longer than the
// fastest of the ten.  The estimate orders them; its own value is further off
// (257 x 14336 -> 4096 28.7 us, measured 22).
inline double line_cost(const Mx4Sizes& a, const SmallTile& t, int cus) {
    const int l = t.a + t.b, pieces = (a.d_in + 255) / 256;
    const double copies = 2 * l + 0.25 * ((l + 1) / 2);
    const int wave_bytes = ln_wave_bytes(t.a, t.b, t.d, t.w);
    const int by_lds = 160 * 1024 / (wave_bytes * t.w), by_waves = (l > 5 ? 16 : 24) / t.w;
    const int together = by_lds < by_waves ? by_lds : by_waves;
    const double tiles = row_tiles(a, 16 * t.a) * ((a.d_out + 16 * t.b - 1) / (16 * t.b));
    const double per_cu = std::ceil(tiles / cus), rounds = std::ceil(per_cu / together);
    const double latency = 1360.0 + (t.d == 2 ? 360.0 : 580.0) * ((pieces + t.w - 1) / t.w) + 6.0 * copies;
    const double work = 13.9 * pieces * copies + 71.0 * t.a * t.b + 570.0;
    const double by_work = per_cu * work + 900.0;
    return 1560.0 + (rounds * latency > by_work ? rounds * latency : by_work);
}
inline double tile_cost(const Mx4Sizes& a, int bm, int bn, int cus) {
    const int pairs = (a.d_in + 511) / 512 * 2;
    const double tiles = row_tiles(a, bm) * ((a.d_out + bn - 1) / bn);
    if (bn == 128) {
        const double full = std::ceil(tiles / (2 * cus)) - 1.0, rest = tiles - full * 2 * cus;
        return full * (1198.0 * pairs + 4270.0) + (rest > cus ? 1198.0 * pairs + 4270.0 : 640.0 * pairs + 4310.0);
    }
    const double rounds = std::ceil(tiles / cus);
    return bm == 128 ? rounds * (970.0 * pairs + 5940.0) + 120.0 : rounds * (1360.0 * pairs + 8630.0) - 500.0;
}
// Short rows (the split kernel): one chunk's latency, and per tile of a CU its
// copies and sums.  0.6% over the fastest of the five at 400 random shapes (1
// to 16384 rows, dense and by up to 64 experts, 32 to 480 inputs, 32 to 16384
// outputs).
inline double split_cost(const Mx4Sizes& a, const SmallTile& t, int cus) {
    const int l = t.a + t.b, copies = l + (l + 3) / 4 * (a.d_in % 128 == 0 ? 1 : 2);
    const double tiles = row_tiles(a, 16 * t.a) * ((a.d_out + 16 * t.b - 1) / (16 * t.b));
    const double work = 16.7 * ((a.d_in + 127) / 128) * copies + 25.5 * t.a * t.b;
    return 3200.0 + 29.0 * copies + 85.0 * t.a * t.b + tiles / cus * work;
}

// The shape with the least estimate.
inline Mx4Pick mx4_pick(const Mx4Sizes& a, int cus) {
    Mx4Pick p{};
    double best = HUGE_VAL;
    auto offer = [&](Mx4Form form, int shape, double cost, int whole) {
        if (cost < best) {
            best = cost;
            p = Mx4Pick{form, shape, a.d_in % whole == 0};
        }
    };
    int id = 0;
    if (a.d_in < kSpRow) {
        for (const SmallTile& t : kSpTiles) offer(Mx4Form::split, id++, split_cost(a, t, cus), 128);
        return p;
    }
    for (const SmallTile& t : kLnTiles) offer(Mx4Form::line, id++, line_cost(a, t, cus), 256);
    // the large tiles take 32-bit offsets into gathered rows
    if (!a.gathered || static_cast<int64_t>(a.n) * (a.d_in / 2) < (int64_t{1} << 32)) {
        id = 0;
        for (const LargeTile& t : kTlTiles) offer(Mx4Form::tile, id++, tile_cost(a, t.bm, t.bn, cus), 512);
    }
    return p;
}

}  // namespace catk
