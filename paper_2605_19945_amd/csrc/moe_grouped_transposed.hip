// Products grouped by expert: rows times transposed weights.
#include "moe_grouped_stream.h"

hipError_t grouped_launch_transposed(const GroupedArgs& g, int bm, hipStream_t st) { return launch_rows<FMT_BF16, LAY_K>(g, bm, st); }
