// Products grouped by expert: the gradient of the weights.
#include "moe_grouped.h"

template <int OUT> static hipError_t launch(const GroupedArgs& g, int bm, hipStream_t st) {
    if (bm == 128) return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 128, 128, 2, 2>(g, st);
    return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 256, 256, 2, 4>(g, st);
}

hipError_t grouped_launch_weights(const GroupedArgs& g, int out, int bm, hipStream_t st) {
    if (out == OUT_F32_ADD) return launch<OUT_F32_ADD>(g, bm, st);
    return out == OUT_F32 ? launch<OUT_F32>(g, bm, st) : launch<OUT_BF16>(g, bm, st);
}
