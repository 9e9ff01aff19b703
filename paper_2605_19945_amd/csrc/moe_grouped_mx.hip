// Launches of the matrix product grouped by expert on microscaled 4-bit operands.
#include "moe_grouped_stream.h"
#include "moe_ops.h"

namespace {

template <int BM, int BN, int WM, int WN> hipError_t launch_tiles(const GroupedArgs& g, hipStream_t st) {
    constexpr int blocks = BM * BN > 128 * 128 ? 256 : 512;
    grouped_tile_kernel<FMT_MX4, LAY_K, LAY_K, OUT_BF16, BM, BN, WM, WN><<<blocks, WM * WN * 64, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_mx(const void* xq, const void* xs, const void* wq, const void* ws, const int32_t* offsets, int rows_cap, int E,
                             int K, int N, void* y, int64_t ldy, hipStream_t st) {
    GroupedArgs g = {};
    g.a = (const char*)xq;
    g.b = (const char*)wq;
    g.sa = (const uint8_t*)xs;
    g.sb = (const uint8_t*)ws;
    g.c = y;
    g.offsets = offsets;
    g.lda = g.ldb = K / 2;
    g.ldc = ldy;
    g.b_expert = (int64_t)K / 2 * N;
    g.E = E;
    g.rows_cap = rows_cap;
    g.N = N;
    g.kbytes = K / 2;
    g.scale_ld = mx_scale_cols(K);
    if (few_rows(rows_cap, E)) return launch_stream<FMT_MX4, LAY_K>(g, st);
    if (rows_cap / E >= 192 && (int64_t)rows_cap / 256 * ((N + 255) / 256) >= 256) return launch_tiles<256, 256, 2, 4>(g, st);
    return launch_tiles<128, 128, 2, 2>(g, st);
}
