// Norm before a block, h = x r w with r = 1 / sqrt(mean(x^2) + eps), and what a block ends with:
//   n = (norm ? y r_y : y) w,  out = scale x + gate n,  h = out r_out w_next.
// Every value is read and written once (4 bytes a value of bf16 for the norm, 8 for the join with the next norm), so memory bounds both.
// The next norm takes the row before it is rounded to the stream's type; each result is rounded once.  Measured: norm of 8191 x 7168 in bf16 49.6 us,
// 4.7 TB/s; join with a row's gate and the next norm of 65536 x 4096 427 us, 5.0 TB/s (a large copy: 5.1); kernels of one row, the norm of 4096
// 2.0 us and the join of 7168 3.7, are a row's latency.
#include "moe_norm.h"

namespace {

// JOIN: there is y (otherwise x is what is normalised).  NEXT: h is wanted.
template <typename S, typename B, int W, int CH, bool JOIN, bool NEXT, bool NT>
__global__ __launch_bounds__(NORM_THREADS) void norm_kernel(NormArgs a) {
    __shared__ float lds[2][8][4];
    constexpr int ROWS = 8 / W;
    const int group = W == 8 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W)), lane = threadIdx.x % (64 * W);
    const int rows = a.n_rows != nullptr ? min(max(*a.n_rows, 0), a.rows) : a.rows;
    const float over_d = 1.f / (float)a.d;
    const Weights<CH> weights(JOIN ? a.w : nullptr, a.w_f32, lane * 8, a.d), weights_next(NEXT ? a.w_next : nullptr, a.w_f32, lane * 8, a.d);
    int turn = 0;
    for (int base = blockIdx.x * ROWS; base < rows; base += gridDim.x * ROWS) {
        const int64_t row = base + group;
        const bool live = row < rows;
        float x[CH][8], y[JOIN ? CH : 1][8], gate = 1.f;
        {
            Eight<S> xw[CH];
            Eight<B> yw[JOIN ? CH : 1];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                const bool here = live && col < a.d;
                xw[c].zero();
                if (here) xw[c].template load<NT>((const S*)a.x + row * a.ldx + col);
                if constexpr (JOIN) {
                    yw[c].zero();
                    if (here) yw[c].template load<NT>((const B*)a.y + row * a.ldy + col);
                }
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                xw[c].open(x[c]);
                if constexpr (JOIN) yw[c].open(y[c]);
            }
        }
        if constexpr (JOIN) {
            float r = 1.f;
            if (a.gate != nullptr && a.ldgate == 0 && live) gate = ((const float*)a.gate)[row];
            if (a.norm) {
                float s[1] = {0.f};
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[0] = fmaf(y[c][j], y[c][j], s[0]);
                group_sums<W>(s, lds, turn);
                r = rsqrtf(fmaf(s[0], over_d, a.eps));
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                if (!(live && col < a.d)) continue;
                float w[8], g[8];
                weights.get(col, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = gate;
                if (a.ldgate != 0) {
                    Eight<B> gw;
                    gw.template load<NT>((const B*)a.gate + row * a.ldgate + col);
                    gw.open(g);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = fmaf(a.scale, x[c][j], g[j] * (y[c][j] * r * w[j]));
                Eight<S>::template store<NT>((S*)a.out + row * a.ldout + col, x[c]);
            }
        }
        if constexpr (NEXT) {
            float s[1] = {0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[0] = fmaf(x[c][j], x[c][j], s[0]);
            group_sums<W>(s, lds, turn);
            const float r = rsqrtf(fmaf(s[0], over_d, a.eps));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                if (!(live && col < a.d)) continue;
                float w[8];
                weights_next.get(col, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = x[c][j] * r * w[j];
                Eight<B>::template store<NT>((B*)a.h + row * a.ldh + col, x[c]);
            }
        }
    }
}

template <typename S, typename B, bool NT> hipError_t launch(const NormArgs& a, hipStream_t st) {
    return with_layout(a.d, [&](auto l) {
        constexpr int W = decltype(l)::W, CH = decltype(l)::CH;
        auto kernel = a.y == nullptr ? norm_kernel<S, B, W, CH, false, true, NT>
                                     : a.h != nullptr ? norm_kernel<S, B, W, CH, true, true, NT> : norm_kernel<S, B, W, CH, true, false, NT>;
        const int groups = (a.rows + 8 / W - 1) / (8 / W);
        kernel<<<groups < 2048 ? groups : 2048, NORM_THREADS, 0, st>>>(a);
        return hipGetLastError();
    });
}

template <typename S, typename B> hipError_t launch(const NormArgs& a, hipStream_t st) {
    const int64_t n = (int64_t)a.rows * a.d, values = a.y == nullptr ? sizeof(S) + sizeof(B) : 2 * sizeof(S) + sizeof(B) * (1 + (a.h != nullptr) + (a.ldgate != 0));
    return norm_streams(n * values) ? launch<S, B, true>(a, st) : launch<S, B, false>(a, st);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
    if (a.x_f32) return a.y_f32 ? launch<float, float>(a, st) : launch<float, uint16_t>(a, st);
    return launch<uint16_t, uint16_t>(a, st);
}
