// Which kernel a product grouped by expert runs on, and into how many ranges its reduction is cut.  Host only; the number of rows
// of each expert is on the device, so the rules go by the bound on the rows and by their mean.  Times in microseconds, fitted to
// calls of 1 to 65536 rows on 1 to 128 experts.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>

struct GroupedPlan {
    int bm;      // rows of a tile: 16, 32 (the streaming kernel), 128, 256 (the tile engine)
    int splits;  // ranges of the reduction; their partial sums need splits * outputs * 4 bytes of workspace
    bool tail;   // the reductions of the last round's tiles (256 rows) may be cut on the device: a slot of workspace for every workgroup
};

constexpr int GROUPED_MAX_SPLITS = 16;
constexpr size_t GROUPED_MAX_WORKSPACE = (size_t)64 << 20;

// A kernel: `slots` tiles at a time, a unit of a tile's reduction takes idle (few tiles, latency) to idle + load (all slots taken, memory)
// microseconds, its end `store`; it reads `rate` bytes a microsecond at the most.  `least`: units of a tile that are gone through at least
// (those that are not there take no memory).
struct GroupedKernel { int bm, slots; double idle, load, store, rate; int least; };

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Experts that have rows, on average over rows that pick one each (against min(rows, E): 32 experts, 13624 to 1600, 32 rows 187 -> 162 us).
static inline int grouped_experts(int rows, int E) { return E == 1 || rows < 1 ? 1 : (int)(E * (1.0 - pow(1.0 - 1.0 / E, rows)) + 0.5); }

// Bytes of workspace a plan needs.
static inline size_t grouped_workspace(const GroupedPlan& p, int64_t outputs) { return p.tail ? (size_t)256 * 256 * 256 * 4 : p.splits > 1 ? (size_t)p.splits * outputs * 4 : 0; }

// The fastest cut of `tiles` tiles of `units` units each: a cut costs a second launch and a way to memory and back for its partial
// sums (one token's reduction of 14336 over 512 columns: 71 us in one piece, 37, 23, 17, 15 in 2, 4, 8, 16; one of 1024 over 1024
// columns 9, in two pieces 12).  Returns its time.
// ragged: the number of tiles is an estimate, and the last round is half full on average.
static inline double grouped_cut(const GroupedKernel& k, int64_t tiles, int64_t units, int64_t outputs, double bytes, int most, bool ragged, int* splits) {
    double best = 0;
    *splits = 1;
    for (int s = 1; s <= most && s <= units; ++s) {
        const double sums = s > 1 ? 4.0 + 2e-6 * s * (double)outputs : 0;
        if (s > 1 && (sums >= best || (size_t)s * outputs * 4 > GROUPED_MAX_WORKSPACE || tiles * (s - 1) >= 2 * k.slots)) break;
        const double rounds = (double)(tiles * s) / k.slots, piece = (double)(((int)units + s - 1) / s);
        const double full = (double)(int64_t)rounds, rest = rounds - full;
        // the end of a tile: bf16 results of a streamed one leave under the next one's loads, but for the last; 32 bits do not
        const double end = (piece < k.least ? k.idle * (k.least - piece) : 0) + (s > 1 && k.store < 2 ? 2 : k.store);
        double t = sums + (s == 1 && k.store < 2 ? 2 : 0) + full * (piece * (k.idle + k.load) + end);
        if (ragged && full > 0) t += rest * (piece * (k.idle + k.load) + end) + 0.5 * piece * k.idle;
        else if (rest > 0) t += piece * (k.idle + k.load * rest) + end;
        if (t < sums + bytes / k.rate) t = sums + bytes / k.rate;
        if (s > 1 && t < 6.5) t = 6.5;  // (the host's second launch)
        if (s == 1 || t < best) {
            best = t;
            *splits = s;
        }
    }
    return best;
}

// Products over ragged rows.  kbytes: of a row of the reduction; row_major: bf16 weights [K, N] (tiles of 128 columns where the weights
// are streamed, otherwise 64); mx: 4-bit operands.  An expert has one row tile at least, and half a one is lost on average.
// Measured, 8 experts, 4096 to 14336, us on row tiles of 16 / 32 / 128 / 256: 8 rows an expert 162 / 163 / 180 / 174, 16 230 / 169 / 185 / 175,
// 32 354 / 258 / 196 / 177, 128 989 / 649 / 282 / 200; 4-bit 41 / 42 / 45 / 50, 53 / 45 / 46 / 50, 86 / 70 / 47 / 51, 242 / 172 / 76 / 65;
// 8 experts, 1024 to 1024, 256 rows an expert: - / - / 19 / 20.  Short reductions, which leave most of a streamed tile's stages empty, on 16 or
// 32 / 128: 128 experts, 88 to 3344, transposed, 1309 rows 36 / 17, 60 experts, 64 to 4096, 300 rows 23 / 18, 128 experts, 512 to 2048, 600
// rows 46 / 54.
//
// Tiles of 256 rows with the last round's reductions cut (a piece costs 0.11 us of memory and sum, the second launch and its end 12): surely
// where all tiles together take half the card or less (1 expert, 14336 to 2048, 1500 rows 130 -> 105 us, 8 experts, 14336 to 1024, 3000
// rows 174 -> 125; 5120 to 5120, 512 rows, where it does not pay by this reckoning, 43 -> 61), otherwise for reductions of 60 steps and more in up to
// 12 rounds, where a round is worth the launch (14336 to 4096, 8 experts, two of them leading, 8192 rows 922 -> 845, biased, 4096 rows 561 -> 484,
// 2 experts, 6144 to 6144, 3000 rows 237 -> 211, 8 experts, 5032 to 2016, 8576 rows 257 -> 224; nothing left to cut in a last round of 8192
// to 2048, 5000 rows 177 -> 180; 49 steps, 3128 to 1024, 8965 rows 65 -> 71).
static inline GroupedPlan grouped_rows_plan(int rows, int E, int kbytes, int N, bool row_major, bool mx) {
    GroupedPlan p = {128, 1, false};
    if (rows <= 0) return p;
    const int experts = grouped_experts(rows, E);
    const GroupedKernel kernels[4] = {{16, 256, mx ? 1.2 : 0.63, mx ? 0.73 : 0.72, mx ? 2.0 : 0.2, 5.9e6, mx ? 2 : 3}, {32, 256, mx ? 1.2 : 0.63, mx ? 0.73 : 0.72, mx ? 2.2 : 0.4, 5.9e6, mx ? 1 : 2},
                                      {128, 512, 0.8, 0.4, 2.0, 5.2e6, 2}, {256, 256, 0.9, 0.55, 5.0, 5.2e6, 2}};
    const double bytes = (double)experts * kbytes * N + (double)rows * (kbytes + 2.0 * N);
    double best = 0;
    for (int i = 0; i < 4; ++i) {
        const GroupedKernel& k = kernels[i];
        if (i == 2 && !mx && rows <= 16 * experts && kbytes > 1024) break;  // (a token on 4 experts, 3448 to 1440: streamed in ranges 14, on tiles in ranges 20)
        int64_t row_tiles = rows / k.bm + experts / 2;
        if (row_tiles < experts) row_tiles = experts;
        const bool stream = k.bm < 128;
        const int64_t tiles = row_tiles * ceil_div(N, stream ? (row_major ? 128 : 64) : k.bm);
        const int64_t units = ceil_div(kbytes, stream ? (mx ? 1024 : row_major ? 256 : 512) : 128);
        int splits;
        bool tail = false;
        double t = grouped_cut(k, tiles, units, (int64_t)rows * N, bytes, k.bm < 256 ? GROUPED_MAX_SPLITS : 1, E > 1 && !stream, &splits);
        if (!stream) t += 1.5;  // (the list of tiles: 8 experts, 128 to 512, 128 rows in a graph 5.6 us streamed, 7.1 on tiles)
        if (k.bm == 256 && mx) {
            // (256 of their values are a step, so few reductions are long enough: 28672 to 8192 in 5000 rows 650 -> 639 us, in 3000 434 -> 442)
        } else if (k.bm == 256 && 2 * tiles <= k.slots) {
            for (int64_t s = 2; s <= k.slots / tiles && s <= units / 4; ++s) {
                const double cut = (double)ceil_div(units, s) * (k.idle + k.load * (tiles * s) / k.slots) + k.store + 12.0 + 0.11 * (tiles * s);
                tail = tail || cut < t;
                if (cut < t) t = cut;
            }
        } else if (k.bm == 256) {
            tail = units >= 60 && tiles <= 12 * k.slots && (E > 1 || tiles % k.slots != 0);
        }
        if (i == 0 || t < best) {
            best = t;
            p = {k.bm, splits, tail};
        }
    }
    return p;
}

// Weight gradients [E, M, N] from `rows` rows: a K step of a 256 x 256 tile takes 1.5 us and its stores 7.5, of two 128 x 128 ones at a
// time 1 and 4 (8 experts, 1024 x 1024: 2048 rows 21 and 17 us, 8192 40 and 32; 4096 x 2048 from 4096 rows 98 and 107; 128 experts,
// 3328 x 160 from 29 rows 58 and 71).
static inline GroupedPlan grouped_weights_plan(int rows, int E, int M, int N) {
    GroupedPlan p = {128, 1, false};
    const int64_t t256 = ceil_div(M, 256) * ceil_div(N, 256) * E, t128 = ceil_div(M, 128) * ceil_div(N, 128) * E;
    const int experts = rows < E ? rows : E;
    const int64_t steps = experts > 0 ? ceil_div(ceil_div(rows, experts), 64) : 1;
    const double t = grouped_cut({128, 512, 1.0, 0.0, 4.0, 1e9, 2}, t128, steps, (int64_t)E * M * N, 0, GROUPED_MAX_SPLITS, false, &p.splits);
    if ((t256 < 256 ? 1.0 : (double)t256 / 256) * ((double)steps * 1.5 + 7.5) < t + 1.0) p = {256, 1, false};
    return p;
}
