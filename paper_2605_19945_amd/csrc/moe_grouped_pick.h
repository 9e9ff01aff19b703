// Which kernel a product grouped by expert runs on, and into how many ranges its reduction is cut.  Host only; the number of rows
// of each expert is on the device, so the rules go by the bound and the mean.
#pragma once
#include <stddef.h>
#include <stdint.h>

struct GroupedPlan {
    int bm;      // rows of a tile: 16, 32 (the streaming kernel), 128, 256 (the tile engine)
    int splits;  // ranges of the reduction; their partial sums need splits * outputs * 4 bytes of workspace
};

constexpr int GROUPED_MAX_SPLITS = 16;
constexpr size_t GROUPED_MAX_WORKSPACE = (size_t)64 << 20;

// Ranges so that `tiles` tiles of `steps` steps each give every one of `slots` workgroups work, each range at least `least` steps
// long.
static inline int grouped_splits(int64_t tiles, int steps, int slots, int least, int64_t outputs) {
    int64_t s = tiles > 0 ? slots / tiles : 1;
    if (s > steps / least) s = steps / least;
    if (s > GROUPED_MAX_SPLITS) s = GROUPED_MAX_SPLITS;
    while (s > 1 && (size_t)s * outputs * 4 > GROUPED_MAX_WORKSPACE) --s;
    return s > 1 ? (int)s : 1;
}

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Products over ragged rows.  kbytes: of a row of the reduction; row_major: weights [K, N] (tiles of 128 columns where the weights are
// streamed, otherwise 64).
static inline GroupedPlan grouped_rows_plan(int rows, int E, int kbytes, int N, bool row_major) {
    GroupedPlan p = {128, 1};
    if (rows <= 0) return p;
    const int experts = rows < E ? rows : E;
    const int64_t outputs = (int64_t)rows * N;
    if (rows <= 32 * experts) {  // the weights bound it
        p.bm = rows <= 8 * experts ? 16 : 32;
        const int64_t tiles = ceil_div(N, row_major ? 128 : 64) * experts;
        p.splits = grouped_splits(tiles, (int)ceil_div(kbytes, row_major ? 256 : 512), 256, 4, outputs);
        return p;
    }
    // half a row tile an expert is lost on average
    const int64_t t256 = ceil_div(N, 256) * (rows / 256 + ceil_div(experts, 2)), t128 = ceil_div(N, 128) * (rows / 128 + ceil_div(experts, 2));
    if (rows / experts >= 192 && t256 >= 256) p.bm = 256;
    else p.splits = grouped_splits(t128, (int)ceil_div(kbytes, 128), 512, 8, outputs);
    return p;
}

// Weight gradients [E, M, N] from `rows` rows.
static inline GroupedPlan grouped_weights_plan(int rows, int E, int M, int N) {
    GroupedPlan p = {128, 1};
    const int64_t t256 = ceil_div(M, 256) * ceil_div(N, 256) * E, t128 = ceil_div(M, 128) * ceil_div(N, 128) * E;
    const int experts = rows < E ? rows : E;
    if (t256 >= 256) p.bm = 256;
    else if (experts > 0) p.splits = grouped_splits(t128, (int)ceil_div(rows / experts, 64), 512, 8, (int64_t)E * M * N);
    return p;
}
