// Products grouped by expert: rows times weights, both microscaled 4-bit values.
#include "moe_grouped_stream.h"

hipError_t grouped_launch_mx(const GroupedArgs& g, int bm, hipStream_t st) { return launch_rows<FMT_MX4, LAY_K>(g, bm, st); }
