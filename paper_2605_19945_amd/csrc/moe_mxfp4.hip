// Microscaled 4-bit floating point (blocks of 32 values along the reduction with one power-of-two scale each):
//   e = max(floor(log2 max|x|) - 2, -127),  code = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| 2^-e (ties to the even code, 6 at the most),
//   scale byte = e + 127, 0 for a block of zeros, 255 (not a number) for a block that holds an infinity or a NaN.
// Row r: values q[r][K / 2], two a byte, the lower index in the lower half; scales s[r][S], S = K / 32 up to the next
// multiple of 16, zeros behind the last block.
// Memory bounds these kernels: 2 + 17/32 bytes a bf16 value.  Rounding is the conversion instruction's, which rounds to
// nearest even and saturates.
// Measured: weights [32, 7168, 4096] 450 us = 5.3 TB/s, back to bf16 510 us = 4.7 TB/s (4 of 5 bytes are written), rows [8192, 4096]
// 18 us = 4.7 TB/s (a large copy 5.1 TB/s).
#include "moe_ops.h"

namespace {

constexpr int kThreads = 256;

struct BlockScale {
    float unit;    // 2^e
    uint32_t byte;
};

// From the bits of a block's largest magnitude (an infinity or NaN has the largest bits of all).
static __device__ inline BlockScale block_scale(uint32_t top) {
    const int field = (int)(top >> 23);  // exponent + 127; 0 for zeros and values below 2^-126
    BlockScale b;
    const int byte = max(field - 2, 0);
    b.byte = field == 255 ? 255 : byte;
    b.unit = byte > 0 ? __uint_as_float((uint32_t)byte << 23) : __uint_as_float(1u << 22);  // 2^-127 is below the normal range
    if (top == 0) b.unit = 1.f;
    return b;
}

static __device__ inline uint32_t codes8(const float* v, const BlockScale& b) {
    if (b.byte == 255) return 0;
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], b.unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], b.unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], b.unit, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], b.unit, 3);
    return c;
}

// Rows: four lanes for every scale byte, 8 values a lane; those of the bytes behind the last block have no values and write zeros.
template <bool F32>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const char* x, int64_t ldx, const int32_t* n_rows, int rows, int K, int S,
                                                               uint8_t* q, uint8_t* s) {
    const int n = n_rows != nullptr ? min(max(*n_rows, 0), rows) : rows;
    const uint32_t per = S * 4;  // lanes a row: four for every scale byte, those behind the last block included
    const uint64_t total = (uint64_t)n * per;
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (uint64_t)gridDim.x * kThreads) {
        const int64_t row = i >> 32 ? (int64_t)(i / per) : (int64_t)((uint32_t)i / per);
        const int at = (int)(i - (uint64_t)row * per), blk = at >> 2;
        float v[8];
        uint32_t top = 0;
        const bool live = blk * 32 < K;
        if (live) {
            if (F32) {
                const u32x4_t* p = (const u32x4_t*)(x + (row * ldx + at * 8) * 4);
                const u32x4_t a = p[0], b = p[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = __uint_as_float(a[j]);
                    v[4 + j] = __uint_as_float(b[j]);
                }
            } else {
                const u32x4_t w = *(const u32x4_t*)(x + (row * ldx + at * 8) * 2);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[2 * j] = __uint_as_float(w[j] << 16);
                    v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
        }
        // S is a multiple of 16, so the four lanes of a block are in the loop together
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        if (live) {
            const BlockScale b = block_scale(top);
            *(uint32_t*)(q + row * (K / 2) + at * 4) = codes8(v, b);
            if ((at & 3) == 0) s[row * S + blk] = (uint8_t)b.byte;
        } else if ((at & 3) == 0) {
            s[row * S + blk] = 0;
        }
    }
}

// Weights w[e][K][N] (bf16, row-major) to q[e][N][K / 2], s[e][N][S]: a workgroup takes 256 reduction values (8 blocks, a
// wave each) of 128 columns (two a lane); the codes turn in LDS and leave as 128 bytes a column.
// high: the workgroups of an XCD go through stretches of columns in bands of so many stretches of the reduction (1: all go through the
// columns side by side).
__global__ __launch_bounds__(512) void mx_quantize_weights_kernel(const uint16_t* w, int E, int K, int N, int S, uint32_t high, uint8_t* q,
                                                              uint8_t* s) {
    __shared__ u32x4_t codes[128][9];  // [column][block], one word more than 8: columns on different banks
    __shared__ __attribute__((aligned(8))) uint8_t scales[128][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t nt = (N + 127) / 128, kt = (K + 255) / 256, at = high > 1 ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    if (at >= nt * kt * E) return;
    const uint32_t e = at / (nt * kt), r = at - e * nt * kt, k1 = r / (high * nt) * high, t = r - k1 * nt, h = min(high, kt - k1);
    const int n0 = t / h * 128, k0 = (k1 + t % h) * 256;
    const int blk = k0 / 32 + wave, n = n0 + 2 * lane;
    if (blk * 32 < K && n < N) {
        const uint32_t* p = (const uint32_t*)(w + ((int64_t)e * K + blk * 32) * N + n);
        uint32_t in[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) in[k] = __builtin_nontemporal_load(p + (int64_t)k * (N / 2));  // read once
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t top = 0;
            float v[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                v[k] = __uint_as_float(c ? in[k] & 0xffff0000u : in[k] << 16);
                top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
            }
            const BlockScale b = block_scale(top);
            u32x4_t o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = codes8(v + 8 * j, b);
            codes[2 * lane + c][wave] = o;
            scales[2 * lane + c][wave] = (uint8_t)b.byte;
        }
    } else {  // behind the last block: nothing of q, zero scales
        scales[2 * lane][wave] = 0;
        scales[2 * lane + 1][wave] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 128 * 8; i += 512) {
        const int c = i >> 3, b = i & 7;
        if (n0 + c < N && k0 + b * 32 < K) *(u32x4_t*)(q + ((int64_t)e * N + n0 + c) * (K / 2) + k0 / 2 + b * 16) = codes[c][b];
    }
    const int c = threadIdx.x;
    if (c < 128 && n0 + c < N) {
        uint64_t* to = (uint64_t*)(s + ((int64_t)e * N + n0 + c) * S + k0 / 32);
        to[0] = *(const uint64_t*)scales[c];
        if (k0 + 256 >= K && k0 / 32 + 8 < S) to[1] = 0;  // S is a multiple of 16: an odd last stretch of 8 blocks leaves 8 more bytes
    }
}

// Back to bf16, which holds every such value exactly: 8 values a lane.
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const uint8_t* q, const uint8_t* s, int64_t rows, int K, int S, uint16_t* x,
                                                                 int64_t ldx) {
    const uint32_t per = K / 8;
    const uint64_t total = (uint64_t)rows * per;
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (uint64_t)gridDim.x * kThreads) {
        const int64_t row = i >> 32 ? (int64_t)(i / per) : (int64_t)((uint32_t)i / per);
        const int at = (int)(i - (uint64_t)row * per);
        const uint32_t c = *(const uint32_t*)(q + row * (K / 2) + at * 4);
        const uint32_t byte = s[row * S + (at >> 2)];
        const float unit = byte == 255 ? __uint_as_float(0x7fc00000u) : byte > 0 ? __uint_as_float(byte << 23) : __uint_as_float(1u << 22);
        u32x4_t o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // magnitude m = 0..7 is 0, 0.5, then (1 + (m & 1) / 2) 2^(m / 2 - 1): bits of a float with a one-bit fraction
                const uint32_t code = c >> (8 * j + 4 * h) & 15, m = code & 7;
                const float mag = m < 2 ? 0.5f * (float)m : __uint_as_float((126u << 23) + (m << 22));
                v[h] = (code & 8 ? -mag : mag) * unit;
            }
            const bf16x2_t p = {(__bf16)v[0], (__bf16)v[1]};
            o[j] = __builtin_bit_cast(uint32_t, p);
        }
        *(u32x4_t*)(x + row * ldx + at * 8) = o;
    }
}

int blocks_of(uint64_t lanes) {
    const uint64_t want = (lanes + kThreads - 1) / kThreads;
    return (int)(want < 8192 ? want : 8192);
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, bool f32, int64_t ldx, const int32_t* n_rows, int rows, int K, void* q, void* s, hipStream_t st) {
    const int S = mx_scale_cols(K);
    auto kernel = f32 ? mx_quantize_kernel<true> : mx_quantize_kernel<false>;
    kernel<<<blocks_of((uint64_t)rows * S * 4), kThreads, 0, st>>>((const char*)x, ldx, n_rows, rows, K, S, (uint8_t*)q, (uint8_t*)s);
    return hipGetLastError();
}

hipError_t launch_mx_quantize_weights(const void* w, int E, int K, int N, void* q, void* s, hipStream_t st) {
    const int64_t blocks = (int64_t)((N + 127) / 128) * ((K + 255) / 256) * E;
    // Where 256 bytes of a row that is read or 128 of one that is written are no whole lines, neighbours in both directions share
    // some, and are kept in one L2 (bands of 4: 8 experts, 12896 x 7968 644 -> 570 us, 64 experts, 13408 x 864 563 -> 430; where they are
    // whole lines, 32 experts, 7168 x 4096 472 -> 507).
    const uint32_t high = K % 256 == 0 && N % 64 == 0 ? 1 : 4;
    mx_quantize_weights_kernel<<<(blocks + 7) / 8 * 8, 512, 0, st>>>((const uint16_t*)w, E, K, N, mx_scale_cols(K), high, (uint8_t*)q, (uint8_t*)s);
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const void* q, const void* s, int64_t rows, int K, void* x, int64_t ldx, hipStream_t st) {
    mx_dequantize_kernel<<<blocks_of((uint64_t)rows * (K / 8)), kThreads, 0, st>>>((const uint8_t*)q, (const uint8_t*)s, rows, K,
                                                                                  mx_scale_cols(K), (uint16_t*)x, ldx);
    return hipGetLastError();
}
