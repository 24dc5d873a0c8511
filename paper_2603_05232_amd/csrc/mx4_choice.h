// Which kernel a product of microscaled operands goes to (host).
#pragma once
#include "mx4_common.h"
#include <math.h>

namespace ss {

// The kernel of a product: tiles of 16 or 32 rows of the kernel for few tokens, MX_SHORT + 16 or 32 of mx4_short.hip (rows of MX_SHORT_UNITS and fewer), MX_MID + 32,
// 64 or 128 of mx4_mid.hip, 256 of mx4_tile.hip.  Which is the fastest goes by an estimate of every kernel's time in us: its launch, then the longest of what its workgroups take one after the other (time of a
// unit and of a workgroup's start and end, times workgroups for each compute unit), what the weights take that are read once for every tile of
// rows (MB over MB per us, L2 and memory-side cache), and the weights from HBM.  The group sizes lie on the device: E experts are taken to have R / E rows
// each, and half a tile more.  Constants fitted to the times of all on 137 shapes (R = 1 .. 54000, 1 .. 79 units, 64 .. 37888 channels, 1 to 128
// experts): the choice is 1.02 of the fastest on average, 1.3 at most.  Times of 16 | 32 | MID + 32 | 64 | 128 | 256, us a call of 24 in a graph, over so many sets of
// weights that they come from HBM (a call on weights that the memory-side cache holds, or one alone in a trace, is up to a tenth shorter):
//   1 x 3584 -> 37888          14.0 |  15.3 |  18.4 |  19.1 |   -   |   -       200 x 4096 -> 14336       49.3 |  36.8 |  24.3 | 17.8 | 14.9 | 27.3
//   32 x 3584 -> 37888         24.2 |  19.7 |  20.0 |  19.9 | 26.9 | 25.9       777 x 5003 -> 4099        77.7 |  50.9 |  30.0 | 20.7 | 18.1 | 33.6
//   64 x 3584 -> 4608           7.2 |   7.9 |   7.3 |   7.8 |   9.6 | 22.0       3200 x 4096 -> 4096        183 |   136 |  76.2 | 51.9 | 51.5 | 33.4
//   8192 x 256 -> 512          17.9 |  18.2 |   8.2 |   5.8 |   5.8 | 10.1       4000 x 256 -> 4096        56.9 |  59.7 |  23.4 | 15.3 | 15.2 | 13.7
//   500 rows, 8 experts, 4096 -> 4096   43.8 | 33.6 | 30.4 | 22.5 | 27.4 | 29.7      4000 rows, 64 experts, 2048 -> 1408   61.9 | 62.0 | 36.3 | 32.6 | 39.5 | 39.5
// and of rows of one to four units 16 | 32 | SHORT + 16 | 32 | the best of MID | 256:
//   3 x 436 -> 8870             3.1 |   3.4 |   3.1 |   3.1 |   3.8 |   8.9       1 x 1024 -> 4096          3.0 |   3.2 |   3.5 |  3.6 |  4.3 |  9.7
//   476 x 303 -> 1000           4.4 |   4.3 |   3.4 |   4.0 |   4.0 |  12.6       200 x 512 -> 16384       15.1 |  16.5 |   8.7 |  8.4 |  5.9 | 10.0
//   500 rows, 64 experts, 512 -> 2048   17.4 | 23.4 | 10.6 | 10.0 | 13.7 | 21.4      8000 rows, 64 experts, 256 -> 1024   44.9 | 44.1 | 13.9 | 12.6 | 14.1 | 19.1
//   300 gated rows, 60 experts, 1024 -> 1408   24.0 | 33.2 | 21.2 | 21.9 | 23.8 | 52.4      8000 rows, 16 experts, 512 -> 2048   85 | 82 | 33 | 28 | 24.6 | 21.8
// Ranges of units (the second kernel, its launch and MB of sums: 3.5 us + 0.36 a MB), split over unsplit: 256 x 18944 -> 3584 23.5 | 33.8, 777 x 18944 -> 512 17.8 | 28.0,
// 100 x 14336 -> 4096 15.4 | 22.3; 64 x 4096 -> 4096, whose estimate is against it, 8.7 | 6.1.
// The kernel of 16 rows takes eight wavefronts, two units each ahead, where rows have 16 units and more, otherwise four (1 x 18944 -> 3584 10.3 against 12.4, 32 gated
// rows of 8 experts 4096 -> 14336 83.7 against 88.6; 512 rows of 64 experts, 8 units, 26.4 against 22.2).
constexpr int MX_MID = 1000, MX_SHORT = 2000;
struct mx4_plan { int kernel, ranges; };
inline mx4_plan mx4_choose(int64_t R, int64_t E, int64_t U, int64_t frags, int64_t cus, size_t ws_bytes)
{
    const bool many = E > 1;
    const double used = many ? (double)E * (1.0 - pow(1.0 - 1.0 / (double)E, (double)R)) : 1.0, MB = (double)(frags * U * (MX_FRAGB + MX_FRAGS)) / 1e6;
    const double hbm = used * MB / 5.2, panels = (double)((frags + 3) / 4), wide = (double)((frags + 7) / 8), u = (double)U;
    auto fits = [&](int64_t T, int64_t threads) { return mx4_grid_fits((frags + 3) / 4 * mx4_max_tiles(R, E, T), threads); };
    auto tiles = [&](int64_t T) { return many ? fmax(used, (double)R / (double)T + 0.5 * used) : (double)((R + T - 1) / T); };
    // workgroups of a compute unit one after the other; a last round that only some have counts as much more than its share as the others wait
    auto rounds = [](double x, double more) { const double part = x - floor(x); return x <= 1.0 ? 1.0 : floor(x) + (part > 0.0 ? fmin(1.0, more + part) : 0.0); };
    mx4_plan best = {};
    double time = INFINITY;
    auto offer = [&](mx4_plan p, double us) {
        if (us < time) { best = p; time = us; }
    };
    const struct { int rows; double launch, rate, row, start, unit; } few[] = {{16, 2.52, 8.5, 0.0, 0.39, 0.056}, {32, 2.67, 5.85, 0.18, 0.73, 0.086}};
    for (const auto& f : few) {
        const double t = tiles(f.rows), shares = (double)frags * t / (double)cus;
        offer({f.rows, 1}, f.launch + fmax(fmax(MB * t / f.rate * (many ? 0.94 : 1.0), f.row * u), fmax((f.start + f.unit * u) * (many ? 1.6 : 1.0) * shares, hbm)));
    }
    if (U <= MX_SHORT_UNITS) {
        const struct { int rows; double launch, start, unit, row; } whole[] = {{16, 2.6, 0.07, 0.41, 0.27}, {32, 2.65, 0.07, 0.70, 0.40}};
        for (const auto& s : whole)
            if (fits(s.rows, 256)) offer({MX_SHORT + s.rows, 1}, s.launch + fmax(fmax((s.start + s.unit * u) * (many ? 1.2 : 1.0) * panels * tiles(s.rows) / (double)cus, s.row * u), 1.13 * hbm));
    }
    const struct { int rows; double launch, unit, ends, hbm, more; } mid[] = {{32, 2.29, 0.39, 0.85, 1.13, 0.0}, {64, 1.92, 0.40, 1.27, 1.13, 0.33}, {128, 1.67, 0.56, 2.76, 1.67, 0.39}};
    for (const auto& m : mid) {
        const double w = panels * tiles(m.rows);
        if (!fits(m.rows, 512)) continue;
        for (int r = 1; r <= 16 && r <= U; ++r) {
            if (r > 1 && (mx4_mid_bytes(R, E, frags, m.rows, r) > ws_bytes || w * r > 2.0 * (double)cus)) break;
            const double add = r > 1 ? 3.5 + 0.36 * w * r * (double)m.rows * 512.0 / 1e6 : 0.0;
            offer({MX_MID + m.rows, r}, m.launch + fmax((m.unit * ceil(u / r) + m.ends) * (many ? 1.46 : 1.0) * rounds(w * r / (double)cus, m.more), m.hbm * hbm + 1.0) + add);
        }
    }
    const double all = wide * tiles(256) / (double)cus, full = fmin(1.0, all);
    offer({256, 1}, 3.94 + fmax(rounds(all, 0.31) * (fmax(u, 3.0) * (1.02 + 0.69 * full) + (0.8 + 3.43 * full) * (many ? 1.83 : 1.0)), hbm));
    return best;
}

}  // namespace ss
