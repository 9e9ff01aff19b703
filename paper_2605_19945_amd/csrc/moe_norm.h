// Norms around a block, row by row: what the forward and the backward unit share.
//
// A row is held in the registers of a group of W wavefronts, CH chunks of 8 neighbouring values a lane, so that each of its values is
// read once, whatever is summed over the row before it is used.  A workgroup is 512 lanes: 8 / W rows at a time, then the rows a
// grid further on.  Sums are in 32 bits: over a lane's values, over the 64 lanes, over the group's wavefronts in their order.
#pragma once
#include "moe_ops.h"

constexpr int NORM_THREADS = 512;

// 8 neighbouring values: 16 bytes of bf16, 32 of fp32
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
    static __device__ inline void load(const uint16_t* p, float (&v)[8]) {
        const u32x4_t w = *(const u32x4_t*)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
    static __device__ inline void store(uint16_t* p, const float (&v)[8]) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        u32x4_t w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2_t t = {(__bf16)v[2 * j], (__bf16)v[2 * j + 1]};  // to nearest even
            w[j] = __builtin_bit_cast(uint32_t, t);
        }
        *(u32x4_t*)p = w;
    }
};
template <> struct Eight<float> {
    static __device__ inline void load(const float* p, float (&v)[8]) {
        const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
    }
    static __device__ inline void store(float* p, const float (&v)[8]) {
        *(f32x4_t*)p = f32x4_t{v[0], v[1], v[2], v[3]};
        *(f32x4_t*)(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
    }
};

// Weights are read again for every row, from the caches: in registers they would cost a row's chunk twice over.
static __device__ inline void load_weights(const void* w, bool f32, int col, float (&v)[8]) {
    if (f32) Eight<float>::load((const float*)w + col, v);
    else Eight<uint16_t>::load((const uint16_t*)w + col, v);
}

static __device__ inline float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// Sums over a group of W wavefronts, in every lane.  `turn` counts the reductions of the workgroup: two neighbouring ones use different
// places, so one barrier each is enough.
template <int W, int N> static __device__ inline void group_sums(float (&v)[N], float (*lds)[8][4], int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if (W == 1) return;
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    float(*slot)[4] = lds[turn & 1];
    ++turn;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) slot[wave][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) v[i] += slot[first + w][i];
    }
}

// The layout of a row of d values; calls f(Layout<W, CH>).  Narrow rows a wavefront each, wide ones all eight.
template <int W_, int CH_> struct Layout { static constexpr int W = W_, CH = CH_; };
template <typename F> static inline hipError_t with_layout(int d, F&& f) {
    if (d <= 512) return f(Layout<1, 1>{});
    if (d <= 1024) return f(Layout<1, 2>{});
    if (d <= 2048) return f(Layout<4, 1>{});
    if (d <= 4096) return f(Layout<8, 1>{});
    if (d <= 8192) return f(Layout<8, 2>{});
    return f(Layout<8, 4>{});
}
static inline int norm_rows_per_group(int d) { return d <= 1024 ? 8 : d <= 2048 ? 2 : 1; }
