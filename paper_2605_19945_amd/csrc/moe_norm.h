// Norms around a block, row by row: what the forward and the backward unit share.
//
// A row is held in the registers of a group of W wavefronts, CH chunks of 8 neighbouring values a lane, so that each of its values is
// read once, whatever is summed over the row before it is used.  A workgroup is 512 lanes: 8 / W rows at a time, then the rows a
// grid further on.  Sums are in 32 bits: over a lane's values, over the 64 lanes, over the group's wavefronts in their order.
#pragma once
#include "moe_ops.h"

constexpr int NORM_THREADS = 512;

// 8 neighbouring values as they lie in memory: 16 bytes of bf16, 32 of fp32.  NT: the non-temporal hint, for rows that no cache holds until their
// next use.
template <bool NT> static __device__ inline u32x4_t load_word(const void* p) { return NT ? __builtin_nontemporal_load((const u32x4_t*)p) : *(const u32x4_t*)p; }
template <bool NT> static __device__ inline void store_word(void* p, const u32x4_t& w) {
    if (NT) __builtin_nontemporal_store(w, (u32x4_t*)p);
    else *(u32x4_t*)p = w;
}
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
    u32x4_t w;
    template <bool NT> __device__ inline void load(const uint16_t* p) { w = load_word<NT>(p); }
    __device__ inline void zero() { w = u32x4_t{0, 0, 0, 0}; }
    __device__ inline void hold() { asm volatile("" : "+v"(w)); }  // what was opened before is opened again rather than kept
    __device__ inline void open(float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
    template <bool NT> static __device__ inline void store(uint16_t* p, const float (&v)[8]) {
        typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
        u32x4_t w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bf16x2_t t = {(__bf16)v[2 * j], (__bf16)v[2 * j + 1]};  // to nearest even
            w[j] = __builtin_bit_cast(uint32_t, t);
        }
        store_word<NT>(p, w);
    }
};
template <> struct Eight<float> {
    u32x4_t w[2];
    template <bool NT> __device__ inline void load(const float* p) { w[0] = load_word<NT>(p), w[1] = load_word<NT>(p + 4); }
    __device__ inline void zero() { w[0] = w[1] = u32x4_t{0, 0, 0, 0}; }
    __device__ inline void hold() {}
    __device__ inline void open(float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j >> 2][j & 3]);
    }
    template <bool NT> static __device__ inline void store(float* p, const float (&v)[8]) {
        u32x4_t a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(v[j]), b[j] = __float_as_uint(v[4 + j]);
        store_word<NT>(p, a);
        store_word<NT>(p + 4, b);
    }
};

static __device__ inline void load_weights(const void* w, bool f32, int col, float (&v)[8]) {
    if (w == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 1.f;
    } else if (f32) {
        Eight<float> e;
        e.load<false>((const float*)w + col);
        e.open(v);
    } else {
        Eight<uint16_t> e;
        e.load<false>((const uint16_t*)w + col);
        e.open(v);
    }
}
// A lane's weights: kept where it has one chunk of a row, otherwise read again for every row, from the caches (in registers they would cost as much
// as a row's chunks).
template <int CH> struct Weights {
    static constexpr bool KEPT = CH == 1;
    const void* at;
    bool f32;
    float kept[8];
    __device__ inline Weights(const void* w, bool f32_, int col, int d) : at(w), f32(f32_) {
        if (KEPT && col < d) load_weights(at, f32, col, kept);
    }
    __device__ inline void get(int col, float (&v)[8]) const {
        if (KEPT) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = kept[j];
        } else {
            load_weights(at, f32, col, v);
        }
    }
};

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

// The layout of a row of d values; calls f(Layout<W, CH>): a chunk a lane where eight wavefronts or fewer do for that.  More wavefronts than that leave
// lanes idle (131072 rows of 512, forward and backward: 41 and 80 us by one wavefront a row, 59 and 184 by four), fewer hold more of a row
// each (32768 rows of 2048: 39 and 88 by four wavefronts, 42 and 109 by one; 32 rows of 1024, join and gradients: 3.1 and 7.2 by two, 3.7
// and 10.6 by one; 16384 rows of 4096, its gradients: 137 by eight, 185 by four).
template <int W_, int CH_> struct Layout { static constexpr int W = W_, CH = CH_; };
template <typename F> static inline hipError_t with_layout(int d, F&& f) {
    if (d <= 512) return f(Layout<1, 1>{});
    if (d <= 1024) return f(Layout<2, 1>{});
    if (d <= 2048) return f(Layout<4, 1>{});
    if (d <= 4096) return f(Layout<8, 1>{});
    if (d <= 8192) return f(Layout<8, 2>{});
    return f(Layout<8, 4>{});
}
// Tensors that the last-level cache (256 MB) does not hold until their next use: `bytes` of all that a call reads and writes.  With the hint the join of
// 65536 rows of 1024 (400 MB) takes 93 us, without 103; the norm of as many (268 MB) 45 with and 41 without.
static inline bool norm_streams(int64_t bytes) { return bytes > (int64_t)256 << 20; }
static inline int norm_rows_per_group(int d) { return d <= 512 ? 8 : d <= 1024 ? 4 : d <= 2048 ? 2 : 1; }
