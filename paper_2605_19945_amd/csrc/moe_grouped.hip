// Launches of the matrix products grouped by expert.
#include "moe_grouped_stream.h"
#include "moe_ops.h"

namespace {

// One workgroup a compute unit (two where two fit), in eights so that every XCD has as many.
template <int FMT, int LA, int LB, int OUT, int BM, int BN, int WM, int WN> hipError_t launch_tiles(const GroupedArgs& g, hipStream_t st) {
    constexpr int blocks = BM * BN > 128 * 128 ? 256 : 512;
    grouped_tile_kernel<FMT, LA, LB, OUT, BM, BN, WM, WN><<<blocks, WM * WN * 64, 0, st>>>(g);
    return hipGetLastError();
}

// 256 x 256 tiles where there are enough of them for every compute unit, 128 x 128 ones otherwise.
bool large_tiles(const GroupedArgs& g, bool weights) {
    const int64_t nt = (g.N + 255) / 256;
    if (weights) return g.E * ((g.M + 255) / 256) * nt >= 256;
    return g.rows_cap / g.E >= 192 && g.rows_cap / 256 * nt >= 256;
}

template <int OUT> hipError_t launch_weights(const GroupedArgs& g, hipStream_t st) {
    if (large_tiles(g, true)) return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 256, 256, 2, 4>(g, st);
    return launch_tiles<FMT_BF16, LAY_MN, LAY_MN, OUT, 128, 128, 2, 2>(g, st);
}

}  // namespace

hipError_t launch_grouped_gemm(const void* x, int64_t ldx, const void* w, bool transpose_w, const int32_t* offsets, int rows_cap, int E,
                               int K, int N, void* y, int64_t ldy, hipStream_t st) {
    GroupedArgs g = {};
    g.a = (const char*)x;
    g.b = (const char*)w;
    g.c = y;
    g.offsets = offsets;
    g.lda = ldx * 2;
    g.ldb = (int64_t)(transpose_w ? K : N) * 2;
    g.ldc = ldy;
    g.b_expert = (int64_t)K * N * 2;
    g.E = E;
    g.rows_cap = rows_cap;
    g.N = N;
    g.kbytes = K * 2;
    if (few_rows(rows_cap, E)) return transpose_w ? launch_stream<FMT_BF16, LAY_K>(g, st) : launch_stream<FMT_BF16, LAY_MN>(g, st);
    const bool large = large_tiles(g, false);
    if (transpose_w)
        return large ? launch_tiles<FMT_BF16, LAY_K, LAY_K, OUT_BF16, 256, 256, 2, 4>(g, st)
                     : launch_tiles<FMT_BF16, LAY_K, LAY_K, OUT_BF16, 128, 128, 2, 2>(g, st);
    return large ? launch_tiles<FMT_BF16, LAY_K, LAY_MN, OUT_BF16, 256, 256, 2, 4>(g, st)
                 : launch_tiles<FMT_BF16, LAY_K, LAY_MN, OUT_BF16, 128, 128, 2, 2>(g, st);
}

hipError_t launch_grouped_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets, int rows_cap, int E,
                                int K, int N, void* dw, bool f32, bool add, hipStream_t st) {
    GroupedArgs g = {};
    g.a = (const char*)x;
    g.b = (const char*)dy;
    g.c = dw;
    g.offsets = offsets;
    g.lda = ldx * 2;
    g.ldb = lddy * 2;
    g.ldc = N;
    g.E = E;
    g.rows_cap = rows_cap;
    g.M = K;
    g.N = N;
    if (add) return launch_weights<OUT_F32_ADD>(g, st);
    return f32 ? launch_weights<OUT_F32>(g, st) : launch_weights<OUT_BF16>(g, st);
}
