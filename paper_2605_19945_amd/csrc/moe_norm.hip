// Norm before a block, h = x r w with r = 1 / sqrt(mean(x^2) + eps), and what a block ends with:
//   n = (norm ? y r_y : y) w,  out = scale x + gate n,  h = out r_out w_next.
// Every value is read and written once (4 bytes a value of bf16 for the norm, 8 for the join with the next norm), so memory bounds both.
// The next norm takes the row before it is rounded to the stream's type; each result is rounded once.
#include "moe_norm.h"

namespace {

// JOIN: there is y (otherwise x is what is normalised).  NEXT: h is wanted.
template <typename S, typename B, int W, int CH, bool JOIN, bool NEXT>
__global__ __launch_bounds__(NORM_THREADS) void norm_kernel(NormArgs a) {
    __shared__ float lds[2][8][4];
    constexpr int ROWS = 8 / W;
    const int group = threadIdx.x / (64 * W), lane = threadIdx.x % (64 * W);
    const int rows = a.n_rows != nullptr ? min(max(*a.n_rows, 0), a.rows) : a.rows;
    const float over_d = 1.f / (float)a.d;
    int turn = 0;
    for (int base = blockIdx.x * ROWS; base < rows; base += gridDim.x * ROWS) {
        const int64_t row = base + group;
        const bool live = row < rows;
        float x[CH][8], y[JOIN ? CH : 1][8], gate = 1.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * 64 * W + lane) * 8;
            const bool here = live && col < a.d;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[c][j] = 0.f;
            if (here) Eight<S>::load((const S*)a.x + row * a.ldx + col, x[c]);
            if constexpr (JOIN) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[c][j] = 0.f;
                if (here) Eight<B>::load((const B*)a.y + row * a.ldy + col, y[c]);
            }
        }
        if constexpr (JOIN) {
            float r = 1.f;
            if (a.norm) {
                float s[1] = {0.f};
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[0] = fmaf(y[c][j], y[c][j], s[0]);
                group_sums<W>(s, lds, turn);
                r = rsqrtf(fmaf(s[0], over_d, a.eps));
            }
            if (a.gate != nullptr && a.ldgate == 0 && live) gate = ((const float*)a.gate)[row];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                if (!(live && col < a.d)) continue;
                float w[8], g[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.f, g[j] = gate;
                if (a.w != nullptr) load_weights(a.w, a.w_f32, col, w);
                if (a.ldgate != 0) Eight<B>::load((const B*)a.gate + row * a.ldgate + col, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = fmaf(a.scale, x[c][j], g[j] * (y[c][j] * r * w[j]));
                Eight<S>::store((S*)a.out + row * a.ldout + col, x[c]);
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
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.f;
                if (a.w_next != nullptr) load_weights(a.w_next, a.w_f32, col, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] = x[c][j] * r * w[j];
                Eight<B>::store((B*)a.h + row * a.ldh + col, x[c]);
            }
        }
    }
}

template <typename S, typename B> hipError_t launch(const NormArgs& a, hipStream_t st) {
    return with_layout(a.d, [&](auto l) {
        constexpr int W = decltype(l)::W, CH = decltype(l)::CH;
        auto kernel = a.y == nullptr ? norm_kernel<S, B, W, CH, false, true> : a.h != nullptr ? norm_kernel<S, B, W, CH, true, true> : norm_kernel<S, B, W, CH, true, false>;
        const int groups = (a.rows + 8 / W - 1) / (8 / W);
        kernel<<<groups < 2048 ? groups : 2048, NORM_THREADS, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
    if (a.x_f32) return a.y_f32 ? launch<float, float>(a, st) : launch<float, uint16_t>(a, st);
    return launch<uint16_t, uint16_t>(a, st);
}
