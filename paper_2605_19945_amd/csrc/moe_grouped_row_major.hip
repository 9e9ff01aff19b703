// Products grouped by expert: rows times row-major weights.
#include "moe_grouped_stream.h"

hipError_t grouped_launch_row_major(const GroupedArgs& g, int bm, hipStream_t st) { return launch_rows<FMT_BF16, LAY_MN>(g, bm, st); }
