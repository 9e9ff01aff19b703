// Gradients of the norms around a block (moe_norm.hip).  With o the row that the next norm took, p = dh w_next, r its factor:
//   D = dout + r (p - o r^2 mean(p o)),  dx = scale D,  dw_next = sum over rows of dh o r;
// and of the join, with n = y r_y w, dn = gate D and q = dn w:
//   dy = r_y (q - y r_y^2 mean(q y))  (without a norm: q),  dw = sum over rows of dn y r_y,  dgate = D n (its row's sum where the gate is a
//   row's number).
// A row's factors come from the rows themselves again, in the same sums as the means, so the forward pass leaves nothing but its
// results.  Memory bounds it: a norm's over 8192 x 2048 of an fp32 stream, with the residual's gradient added, 49.3 us, 4.8 TB/s; a join's over
// 8192 x 4096 with a gate of values and the next norm's 99.9 us, 5.4 TB/s (second kernel counted).  The gradients of weights are summed over a workgroup's rows in registers, over the workgroup in LDS and
// over the workgroups by a second kernel, each in a fixed order.
#include "moe_norm.h"

namespace {

// A lane's chunks of one row
template <typename S, typename B, int CH, bool JOIN, bool NEXT> struct Row {
    Eight<S> D[CH], o[NEXT ? CH : 1];
    Eight<B> dh[NEXT ? CH : 1], y[JOIN ? CH : 1], g[JOIN ? CH : 1];
    float gate;
};

template <typename S, typename B, int W, int CH, bool JOIN, bool NEXT, bool NT>
__global__ __launch_bounds__(NORM_THREADS, CH * (sizeof(S) + sizeof(B)) <= 6 ? 4 : 2) void norm_backward_kernel(NormGradArgs a) {
    __shared__ float lds[2][8][4];
    extern __shared__ float sums[];  // [d] where a workgroup has several rows
    constexpr int ROWS = 8 / W;
    constexpr bool AHEAD = !(JOIN && NEXT) && CH * (sizeof(S) + sizeof(B)) <= 8;  // the next row is asked for before this one is summed (where registers are left)
    const int group = W == 8 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * W)), lane = threadIdx.x % (64 * W);
    const int rows = a.n_rows != nullptr ? min(max(*a.n_rows, 0), a.rows) : a.rows;
    const float over_d = 1.f / (float)a.d;
    const Weights<CH> weights(JOIN ? a.w : nullptr, a.w_f32, lane * 8, a.d), weights_next(NEXT ? a.w_next : nullptr, a.w_f32, lane * 8, a.d);
    float dw[JOIN ? CH : 1][8] = {}, dnext[NEXT ? CH : 1][8] = {};
    int turn = 0;
    auto fetch = [&](Row<S, B, CH, JOIN, NEXT>& f, int base) {
        const int64_t row = base + group;
        const bool live = row < rows;
        f.gate = 1.f;
        if (JOIN && a.gate != nullptr && a.ldgate == 0 && live) f.gate = ((const float*)a.gate)[row];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * 64 * W + lane) * 8;
            const bool here = live && col < a.d;
            f.D[c].zero();
            if (here && a.dout != nullptr) f.D[c].template load<NT>((const S*)a.dout + row * a.lddout + col);
            if constexpr (NEXT) {
                f.o[c].zero(), f.dh[c].zero();
                if (here) f.o[c].template load<NT>((const S*)a.o + row * a.ldo + col), f.dh[c].template load<NT>((const B*)a.dh + row * a.lddh + col);
            }
            if constexpr (JOIN) {
                f.y[c].zero(), f.g[c].zero();
                if (here) f.y[c].template load<NT>((const B*)a.y + row * a.ldy + col);
                if (here && a.ldgate != 0) f.g[c].template load<NT>((const B*)a.gate + row * a.ldgate + col);
            }
        }
    };
    auto open_gate = [&](const Row<S, B, CH, JOIN, NEXT>& f, int c, float (&g)[8]) {
        if (a.ldgate != 0) {
            f.g[c].open(g);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = 1.f;
        }
    };
    Row<S, B, CH, JOIN, NEXT> next;
    if (AHEAD) fetch(next, blockIdx.x * ROWS);
    for (int base = blockIdx.x * ROWS; base < rows; base += gridDim.x * ROWS) {
        const int64_t row = base + group;
        const bool live = row < rows;
        if (!AHEAD) fetch(next, base);
        Row<S, B, CH, JOIN, NEXT> f = next;
        if (AHEAD) fetch(next, base + gridDim.x * ROWS);  // (behind the last row: nothing)
        float s[3] = {0.f, 0.f, 0.f};  // sums of o^2, p o and y^2
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * 64 * W + lane) * 8;
            if constexpr (NEXT) {
                float w[8] = {}, o[8], dh[8];
                if (col < a.d) weights_next.get(col, w);
                f.o[c].open(o), f.dh[c].open(dh);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[0] = fmaf(o[j], o[j], s[0]);
                    s[1] = fmaf(dh[j] * w[j], o[j], s[1]);
                }
                f.o[c].hold(), f.dh[c].hold();
            }
            if constexpr (JOIN) {
                float y[8];
                f.y[c].open(y);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[2] = fmaf(y[j], y[j], s[2]);
                f.y[c].hold();
            }
        }
        if (NEXT || a.norm) group_sums<W>(s, lds, turn);
        // o r^2 mean(p o) as (o r) (r mean(p o)), factors of p's size: r^3 leaves the range at rows of 1e-13 and 1e13
        const float r = rsqrtf(fmaf(s[0], over_d, a.eps)), k = r * (s[1] * over_d);
        const float ry = JOIN && a.norm ? rsqrtf(fmaf(s[2], over_d, a.eps)) : 1.f;
        float u[1] = {0.f};  // sum of g D w y, without the row's gate
        float D[JOIN ? CH : 1][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * 64 * W + lane) * 8;
            if (!(live && col < a.d)) continue;
            float* Dc = D[JOIN ? c : 0];
            float out[8];
            f.D[c].open(out);
            if constexpr (NEXT) {
                float w[8], o[8], dh[8];
                weights_next.get(col, w);
                f.o[c].open(o), f.dh[c].open(dh);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    out[j] = fmaf(r, dh[j] * w[j] - o[j] * r * k, out[j]);
                    dnext[c][j] = fmaf(dh[j], o[j] * r, dnext[c][j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                Dc[j] = out[j];
                if (JOIN) out[j] *= a.scale;
            }
            Eight<S>::template store<NT>((S*)a.dx + row * a.lddx + col, out);
            if constexpr (JOIN) {
                float w[8], y[8], g[8];
                weights.get(col, w);
                f.y[c].open(y);
                open_gate(f, c, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[0] = fmaf(g[j] * Dc[j], w[j] * y[j], u[0]);
                if (a.ldgate != 0 && a.dgate != nullptr) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) out[j] = Dc[j] * (y[j] * ry * w[j]);
                    Eight<B>::template store<NT>((B*)a.dgate + row * a.lddgate + col, out);
                }
                f.y[c].hold(), f.g[c].hold();
            }
        }
        if constexpr (JOIN) {
            const bool row_gate = a.ldgate == 0 && a.dgate != nullptr;
            if (a.norm || row_gate) group_sums<W>(u, lds, turn);
            if (row_gate && live && lane == 0) ((float*)a.dgate)[row] = u[0] * ry;
            const float ky = a.norm ? ry * (f.gate * u[0] * over_d) : 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                if (!(live && col < a.d)) continue;
                float w[8], y[8], g[8], out[8];
                weights.get(col, w);
                f.y[c].open(y);
                open_gate(f, c, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float dn = f.gate * g[j] * D[c][j];
                    out[j] = a.norm ? ry * (dn * w[j] - y[j] * ry * ky) : dn * w[j];  // (without a norm y has no part in it, an infinite one neither)
                    dw[c][j] = fmaf(dn, y[j] * ry, dw[c][j]);
                }
                Eight<B>::template store<NT>((B*)a.dy + row * a.lddy + col, out);
            }
        }
    }
    // the workgroup's sums, its groups in their order
    auto leave = [&](float (*v)[8], float* part) {
        part += (int64_t)blockIdx.x * a.d;
        if constexpr (ROWS > 1) {
            for (int i = 0; i < ROWS; ++i) {
                if (group == i) {
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        const int col = (c * 64 * W + lane) * 8;
                        if (col >= a.d) continue;
                        float t[8] = {};
                        if (i > 0) load_weights(sums, true, col, t);
#pragma unroll
                        for (int j = 0; j < 8; ++j) t[j] += v[c][j];
                        Eight<float>::store<false>((i < ROWS - 1 ? sums : part) + col, t);
                    }
                }
                __syncthreads();
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * 64 * W + lane) * 8;
                if (col < a.d) Eight<float>::store<false>(part + col, v[c]);
            }
        }
    };
    if (JOIN && a.dw_part != nullptr) leave(dw, a.dw_part);
    if (NEXT && a.dnext_part != nullptr) leave(dnext, a.dnext_part);
}

// dw = the sum of the workgroups' rows: 64 columns a workgroup, 16 lanes of 4 across and 16 ranges of the rows down, joined in LDS.
__global__ __launch_bounds__(256) void norm_weights_kernel(const float* part0, float* out0, const float* part1, float* out1, int n, int d) {
    __shared__ f32x4_t lds[16][16];
    const float* part = blockIdx.y == 0 ? part0 : part1;
    float* out = blockIdx.y == 0 ? out0 : out1;
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4, col = blockIdx.x * 64 + x * 4;
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (col < d) {
#pragma unroll 8
        for (int i = y; i < n; i += 16) s += *(const f32x4_t*)(part + (int64_t)i * d + col);
    }
    lds[y][x] = s;
    __syncthreads();
    if (y == 0 && col < d) {
        for (int i = 1; i < 16; ++i) s += lds[i][x];
        *(f32x4_t*)(out + col) = s;
    }
}

template <typename S, typename B, bool NT> hipError_t launch(const NormGradArgs& a, int grid, hipStream_t st) {
    return with_layout(a.d, [&](auto l) {
        constexpr int W = decltype(l)::W, CH = decltype(l)::CH;
        auto kernel = a.y == nullptr ? norm_backward_kernel<S, B, W, CH, false, true, NT>
                                     : a.dh != nullptr ? norm_backward_kernel<S, B, W, CH, true, true, NT> : norm_backward_kernel<S, B, W, CH, true, false, NT>;
        kernel<<<grid, NORM_THREADS, W < 8 ? a.d * 4 : 0, st>>>(a);
        return hipGetLastError();
    });
}

template <typename S, typename B> hipError_t launch(const NormGradArgs& a, int grid, hipStream_t st) {
    const int64_t n = (int64_t)a.rows * a.d, stream = sizeof(S) * (1 + (a.dout != nullptr) + (a.dh != nullptr)),
                  block = sizeof(B) * ((a.dh != nullptr) + (a.y != nullptr ? 2 : 0) + (a.ldgate != 0 ? 2 : 0));
    return norm_streams(n * (stream + block)) ? launch<S, B, true>(a, grid, st) : launch<S, B, false>(a, grid, st);
}

}  // namespace

int norm_grad_groups(int rows, int d) {
    // As many as the compute units hold at once, two each, one of rows that take more than a chunk a lane: more leave a last round in which units
    // idle, and more sums for the second kernel (16384 rows of 4096, the norm's gradients: 81 us in 512, 89 in 1024, 117 in 256;
    // 2048 rows of 8192, the join's: 50 in 256, 56 in 512, 65 in 1024).
    const int per = norm_rows_per_group(d), want = (rows + per - 1) / per, most = d <= 4096 ? 512 : 256;
    return want < most ? want : most;
}

hipError_t launch_norm_backward(NormGradArgs a, float* dw, float* dw_next, float* workspace, hipStream_t st) {
    const int grid = norm_grad_groups(a.rows, a.d);
    const bool both = dw != nullptr && dw_next != nullptr;
    a.dw_part = dw != nullptr ? workspace : nullptr;
    a.dnext_part = dw_next != nullptr ? workspace + (both ? (int64_t)grid * a.d : 0) : nullptr;
    if (grid > 0) {
        const hipError_t e = a.x_f32 ? (a.y_f32 ? launch<float, float>(a, grid, st) : launch<float, uint16_t>(a, grid, st)) : launch<uint16_t, uint16_t>(a, grid, st);
        if (e != hipSuccess || (dw == nullptr && dw_next == nullptr)) return e;
    }
    if (dw == nullptr && dw_next == nullptr) return hipSuccess;
    const float* p0 = dw != nullptr ? a.dw_part : a.dnext_part;
    norm_weights_kernel<<<dim3((a.d + 63) / 64, both ? 2 : 1), 256, 0, st>>>(p0, dw != nullptr ? dw : dw_next, a.dnext_part, dw_next, grid, a.d);
    return hipGetLastError();
}
