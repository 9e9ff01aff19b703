// Products grouped by expert: the gradient of the weights.
#include "moe_grouped.h"

template <int OUT, bool LINES> static hipError_t launch_lines(const GroupedArgs& g, int bm, hipStream_t st) {
    if (bm == 128) return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 128, 128, 2, 2, false, LINES>(g, st);
    return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 256, 256, 2, 4, false, LINES>(g, st);
}

// Rows that begin at multiples of 64 bytes are written in whole units of memory and take the non-temporal hint; others share units
// with their neighbours, which only a cache can put together.  With the hint and without, us: 128 experts, 2048 x 1528 in fp32 from 65528
// rows 768 and 740, 60 experts, 1408 x 2056 in bf16 from 9000 184 and 154, 8 experts, 12816 x 4488 from 113 466 and 260; at multiples of
// 64, 60 experts, 1408 x 2080 from 9000 113 and 161, 16 experts, 2048 x 5136 in fp32 from 4000 181 and 254, 32 experts, 3288 x 3552
// with next to no rows 196 and 176.
template <int OUT> static hipError_t launch(const GroupedArgs& g, int bm, hipStream_t st) {
    const bool lines = ((uintptr_t)g.c | (uint64_t)g.ldc * (OUT == OUT_BF16 ? 2 : 4)) % 64 == 0;
    return lines ? launch_lines<OUT, true>(g, bm, st) : launch_lines<OUT, false>(g, bm, st);
}

hipError_t grouped_launch_weights(const GroupedArgs& g, int out, int bm, hipStream_t st) {
    if (out == OUT_F32_ADD) return launch<OUT_F32_ADD>(g, bm, st);
    return out == OUT_F32 ? launch<OUT_F32>(g, bm, st) : launch<OUT_BF16>(g, bm, st);
}
