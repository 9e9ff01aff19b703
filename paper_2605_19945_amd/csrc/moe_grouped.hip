// Launches of the matrix products grouped by expert.
#include "moe_grouped.h"
#include "moe_ops.h"

namespace {

// Partial sums of the ranges of a reduction, added in their order: the rows that belong to an expert ...
__global__ __launch_bounds__(256) void sum_rows_kernel(GroupedArgs g) {
    const int per = g.N / 8;  // lanes a row
    for (int e = blockIdx.y; e < g.E; e += gridDim.y) {
        int lo, n;
        expert_rows(g.offsets, e, g.rows_cap, &lo, &n);
        const int64_t total = (int64_t)n * per;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
            const int64_t row = lo + i / per;
            const int col = (int)(i % per) * 8;
            const float* from = g.part + row * g.N + col;
            f32x4_t u = *(const f32x4_t*)from, v = *(const f32x4_t*)(from + 4);
            for (int s = 1; s < g.splits; ++s) {
                u += *(const f32x4_t*)(from + s * g.slab);
                v += *(const f32x4_t*)(from + s * g.slab + 4);
            }
            *(u32x4_t*)((uint16_t*)g.c + row * g.ldc + col) = u32x4_t{pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
    }
}

// ... and the weights (accumulated: of the experts that have rows).
template <int OUT> __global__ __launch_bounds__(256) void sum_weights_kernel(GroupedArgs g) {
    const int64_t per = (int64_t)g.M * g.N / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per * g.E; i += (int64_t)gridDim.x * 256) {
        if (OUT == OUT_F32_ADD) {
            int lo, n;
            expert_rows(g.offsets, (int)(i / per), g.rows_cap, &lo, &n);
            if (n == 0) continue;
        }
        const float* from = g.part + i * 8;
        f32x4_t u = *(const f32x4_t*)from, v = *(const f32x4_t*)(from + 4);
        for (int s = 1; s < g.splits; ++s) {
            u += *(const f32x4_t*)(from + s * g.slab);
            v += *(const f32x4_t*)(from + s * g.slab + 4);
        }
        if (OUT == OUT_BF16) {
            ((u32x4_t*)g.c)[i] = u32x4_t{pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        } else {
            f32x4_t* to = (f32x4_t*)g.c + 2 * i;
            to[0] = OUT == OUT_F32_ADD ? to[0] + u : u;
            to[1] = OUT == OUT_F32_ADD ? to[1] + v : v;
        }
    }
}

// The cut tiles of the last round (256 x 256; a workgroup adds 32 rows of one): the sums of its ranges in their order.
__global__ __launch_bounds__(256) void sum_pieces_kernel(GroupedArgs g) {
    __shared__ TileList list;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nt = (g.N + 255) / 256;
    if (wave == 0) make_list<false, 256, true>(g, nt, &list);
    __syncthreads();
    const int pieces = list.pieces, rest = list.rest, unit = blockIdx.x >> 3;
    if (pieces == 1 || unit >= 8 * rest) return;
    const int j = unit >> 3;
    const GroupedTile t = find_tile<false, 256, 256, true>(g, list, 1, list.height, 0, nt, list.whole + j);
    const int row0 = (unit & 7) * 32 + wave * 8, col = lane * 4, rows = t.rows - row0;
    if (rows <= 0 || col >= g.N - t.n0) return;
    const float* from = g.part + ((blockIdx.x & 7) * SIDE + j) * PIECE + row0 * 256 + col;
    f32x4_t sum[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) sum[r] = r < rows ? *(const f32x4_t*)(from + r * 256) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int s = 1; s < pieces; ++s) {
        const float* p = from + s * rest * PIECE;
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < rows) sum[r] += *(const f32x4_t*)(p + r * 256);
    }
    uint16_t* to = (uint16_t*)g.c + ((int64_t)t.lo + t.m0 + row0) * g.ldc + t.n0 + col;
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (r < rows) *(uint2*)(to + r * g.ldc) = uint2{pack_bf16(sum[r][0], sum[r][1]), pack_bf16(sum[r][2], sum[r][3])};
}

int blocks_of(int64_t lanes) {
    const int64_t want = ceil_div(lanes, 256);
    return (int)(want < 2048 ? want : 2048);
}

// A plan carried out: the product, and the sum of its ranges if its reduction was cut.
template <typename L> hipError_t run_rows(GroupedArgs& g, const GroupedPlan& p, void* ws, hipStream_t st, L launch) {
    g.splits = p.splits;
    g.slab = (int64_t)g.rows_cap * g.N;
    g.part = (float*)(p.splits > 1 || p.tail ? ws : nullptr);
    const hipError_t e = launch(g, p.bm, st);
    if (e != hipSuccess || g.part == nullptr) return e;
    if (p.tail) {
        sum_pieces_kernel<<<8 * 8 * SIDE / 2, 256, 0, st>>>(g);
        return hipGetLastError();
    }
    const int experts = g.rows_cap < g.E ? g.rows_cap : g.E;
    sum_rows_kernel<<<dim3(blocks_of(ceil_div(g.rows_cap, experts) * (g.N / 8)), g.E), 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_gemm(const void* x, int64_t ldx, const void* w, bool transpose_w, const int32_t* offsets, int rows_cap, int E,
                               int K, int N, void* y, int64_t ldy, const GroupedPlan& plan, void* ws, hipStream_t st) {
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
    return run_rows(g, plan, ws, st, transpose_w ? grouped_launch_transposed : grouped_launch_row_major);
}

hipError_t launch_grouped_mx(const void* xq, const void* xs, const void* wq, const void* wsc, const int32_t* offsets, int rows_cap, int E,
                             int K, int N, void* y, int64_t ldy, const GroupedPlan& plan, void* ws, hipStream_t st) {
    GroupedArgs g = {};
    g.a = (const char*)xq;
    g.b = (const char*)wq;
    g.sa = (const uint8_t*)xs;
    g.sb = (const uint8_t*)wsc;
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
    return run_rows(g, plan, ws, st, grouped_launch_mx);
}

hipError_t launch_grouped_wgrad(const void* x, int64_t ldx, const void* dy, int64_t lddy, const int32_t* offsets, int rows_cap, int E,
                                int K, int N, void* dw, bool f32, bool add, const GroupedPlan& plan, void* ws, hipStream_t st) {
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
    g.splits = plan.splits;
    g.slab = (int64_t)E * K * N;
    g.part = (float*)ws;
    const int out = add ? OUT_F32_ADD : f32 ? OUT_F32 : OUT_BF16;
    const hipError_t e = grouped_launch_weights(g, out, plan.bm, st);
    if (e != hipSuccess || g.splits == 1) return e;
    auto kernel = add ? sum_weights_kernel<OUT_F32_ADD> : f32 ? sum_weights_kernel<OUT_F32> : sum_weights_kernel<OUT_BF16>;
    kernel<<<blocks_of((int64_t)E * K * N / 8), 256, 0, st>>>(g);
    return hipGetLastError();
}
