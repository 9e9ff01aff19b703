// Stacks of matrices brought near the orthogonal matrices next to them by Newton-Schulz steps:
//   X = G / (|G| + eps);  for each step (a, b, c):  S = X X^T,  P = b S + c S S,  X = a X + P X;  out = scale X.
// (tall matrices: the same on the transpose).  Singular vectors stay, and each singular value s goes through a s + b s^3 + c s^5.
//
// Products bound it: of n x m matrices, n <= m, n n m + n n n + 2 n n m operations a step where the two symmetric products are formed on
// and above the diagonal only.  Matrix instructions take 16-bit operands, and what a step rounds is multiplied by the ones behind it (by a
// each, for the small singular values), so operands are kept in one or two parts of fp16 (moe_orth.h).  For an fp32 result all of them have
// two: 22 bits, results as far from the exact ones as those of 32-bit products (4e-7 to 2e-6 of their norm, on flat and steep spectra).
// For a bf16 result X where it is multiplied by P, and S, have two, X in S and P one: 2e-5 to 1.2e-3 of the norm, below the 1.7e-3 of
// the result's own rounding; with one part throughout steep spectra lose 8e-3, in bf16 6e-2.
//
// S = X X^T wants X with the reduction along m, P X wants it along n: the epilogue of the last product of a step writes X and X^T.
#include "moe_orth.h"

namespace {

// X, S and P are held times these powers of two: in the middle of fp16's range, singular values up to 4 allowed for, so that the
// second parts are seldom subnormal.
constexpr float X_SCALE = 8192.f, S_SCALE = 4096.f, P_SCALE = 4096.f;

// ---- the products ----
// Tile t of a symmetric matrix's mt x mt, row by row on and above the diagonal
static __device__ inline void place_symmetric(int t, int mt, int* m, int* n) {
    int r = (int)(((2 * mt + 1) - sqrtf((float)((2 * mt + 1) * (2 * mt + 1) - 8 * t))) * 0.5f);
    r = max(min(r, mt - 1), 0);
    while (r > 0 && r * mt - r * (r - 1) / 2 > t) --r;
    while ((r + 1) * mt - (r + 1) * r / 2 <= t) ++r;
    *m = r;
    *n = r + t - (r * mt - r * (r - 1) / 2);
}

// PA, PB: parts of A and B.  WM x WN wavefronts of FM x FN fragments (16 x 16).  STAGES of 32 values of the reduction in LDS: the next
// ones but one arrive while one is multiplied.  CIN: parts of what beta multiplies (0: none).  OUT: parts of the result in blocks (1, 2) or
// its type in the caller's rows.  SYM: the result is symmetric; tiles above the diagonal are written to both sides.
template <int PA, int PB, int WM, int WN, int FM, int FN, int KS, int STAGES, int CIN, int PARTS, int OUT>
__global__ __launch_bounds__(WM* WN * 64) void orth_product_kernel(OrthArgs g) {
    constexpr int WAVES = WM * WN, FA = WM * FM, FB = WN * FN, FRAGS = KS * (FA * PA + FB * PB), LOADS = FRAGS / WAVES;
    static_assert(FA % WAVES == 0 && FB % WAVES == 0, "a load's operand does not depend on the wavefront");
    constexpr bool SYM = OUT == ORTH_SQUARE;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // neighbouring tiles on one XCD (workgroup number % 8): one stretch of the list each
    const int total = g.tiles * g.matrices, xcd = blockIdx.x & 7, each = total >> 3, rest = total & 7;
    const int item = xcd * each + min(xcd, rest) + (blockIdx.x >> 3);
    const int matrix = item / g.tiles, t = item - matrix * g.tiles;
    int tm, tn;
    if constexpr (SYM) {
        place_symmetric(t, g.mt, &tm, &tn);
    } else {  // bands of 8 tiles
        const int band = t / (8 * g.nt), r = t - band * 8 * g.nt, h = min(8, g.mt - 8 * band);
        tn = r / h;
        tm = 8 * band + r - tn * h;
    }
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);

    // loads: block row i * WAVES + wave of the operand that load i belongs to
    const uint32_t panel = (uint32_t)g.steps * ORTH_BLOCK;
    u32x4_t da[PA], db[PB];
#pragma unroll
    for (int p = 0; p < PA; ++p) da[p] = orth_desc(g.a.part[p] + matrix * g.a.matrix + (int64_t)tm * FA * panel, FA * panel);
#pragma unroll
    for (int p = 0; p < PB; ++p) db[p] = orth_desc(g.b.part[p] + matrix * g.b.matrix + (int64_t)tn * FB * panel, FB * panel);
    constexpr int ROUNDS = (FA > FB ? FA : FB) / WAVES;
    uint32_t offset[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) offset[i] = (uint32_t)(i * WAVES + wave) * panel + lane * 16;
    const uint32_t base = __builtin_amdgcn_readfirstlane(orth_lds_addr(lds)) + wave * ORTH_BLOCK;
    constexpr int NA = FA / WAVES, NB = FB / WAVES, PER = PA * NA + PB * NB;  // loads of a block of the reduction
    auto issue_one = [&](auto load, int s, int place) {  // one load of stage s
        constexpr int k = decltype(load)::value / PER, i = decltype(load)::value % PER, ib = i - PA * NA;
        const uint32_t to = base + place * (FRAGS * ORTH_BLOCK), at = (uint32_t)(s * KS + k) * ORTH_BLOCK;
        if constexpr (i < PA * NA) orth_load(to + (KS * (i / NA) * FA + k * FA + i % NA * WAVES) * ORTH_BLOCK, offset[i % NA], da[i / NA], at);
        else orth_load(to + (KS * (PA * FA + ib / NB * FB) + k * FB + ib % NB * WAVES) * ORTH_BLOCK, offset[ib % NB], db[ib / NB], at);
    };
    auto issue = [&](int s, int place) { orth_repeat<LOADS>([&](auto load) { issue_one(load, s, place); }); };

    f32x4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    if constexpr (WAVES == 8) {
        // Two groups of four wavefronts, one of each on every SIMD, take turns: while one group multiplies, the other reads its next
        // fragments, so the matrix cores always have a wavefront whose operands are there.  In turn 2 s the first group reads stage s (and
        // asks for stage s + 1, into the place that the second group left in the turn before), in 2 s + 1 the second; a stage has two turns to
        // arrive.
        f16x8_t a[KS][PA][FM], b[KS][PB][FN];
        const int stages = g.steps / KS;
        auto read = [&](int s) {
            const char* at = lds + (s & 1) * (FRAGS * ORTH_BLOCK) + lane * 16;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
#pragma unroll
                for (int p = 0; p < PB; ++p)
#pragma unroll
                    for (int j = 0; j < FN; ++j) b[k][p][j] = *(const f16x8_t*)(at + (KS * (PA * FA + p * FB) + k * FB + wn * FN + j) * ORTH_BLOCK);
#pragma unroll
                for (int p = 0; p < PA; ++p)
#pragma unroll
                    for (int i = 0; i < FM; ++i) a[k][p][i] = *(const f16x8_t*)(at + (KS * p * FA + k * FA + wm * FM + i) * ORTH_BLOCK);
            }
        };
        constexpr int PAIRS = PA + PB - 1, ROWS = KS * PAIRS * FM;  // rows of fragments that a stage's products come in
        auto multiply = [&](auto&& beside) {
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            orth_repeat<ROWS>([&](auto row) {
                constexpr int k = decltype(row)::value / (PAIRS * FM), pair = decltype(row)::value / FM % PAIRS, i = decltype(row)::value % FM;
                constexpr int p = pair < PB ? 0 : 1, q = pair < PB ? pair : 0;  // hi hi, hi lo, lo hi
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[k][q][j], a[k][p][i], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                beside(row);
            });
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };
        issue(0, 0);
        orth_wait<0>();
        orth_barrier();
        if (wave < 4) {
            for (int s = 0; s < stages; ++s) {
                read(s);
                if (s + 1 < stages) issue(s + 1, (s + 1) & 1);
                orth_barrier();
                multiply([](auto) {});
                orth_wait<0>();
                orth_barrier();
            }
            orth_barrier();
        } else {
            if (1 < stages) issue(1, 1);
            orth_barrier();
            for (int s = 0; s < stages; ++s) {
                read(s);
                orth_wait<0>();
                orth_barrier();
                const bool more = s + 2 < stages;
                multiply([&](auto row) {  // its loads among the products
                    constexpr int r = decltype(row)::value;
                    if constexpr (r * LOADS % ROWS < LOADS && r * LOADS / ROWS < LOADS) {
                        if (more) issue_one(OrthInt<r * LOADS / ROWS>{}, s + 2, s & 1);
                    }
                });
                orth_barrier();
            }
        }
    } else {
        static_assert(WAVES == 8 || KS == 1, "");
        const int stages = g.steps;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (s < stages) issue(s, s);
        int stage = 0;
        for (int step = 0; step < stages; ++step) {
            // this step's stage has arrived; the last steps have fewer behind them and wait for all
            if (step + STAGES - 1 <= stages) orth_wait<(STAGES - 2) * LOADS>();
            else orth_wait<0>();
            orth_barrier();  // of every wavefront's; and all are done with the stage before
            if (step + STAGES - 1 < stages) issue(step + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
            const char* at = lds + stage * (FRAGS * ORTH_BLOCK) + lane * 16;
            const char* fa = at + wm * FM * ORTH_BLOCK;
            const char* fb = at + (PA * FA + wn * FN) * ORTH_BLOCK;
            f16x8_t b[PB][FN];
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int j = 0; j < FN; ++j) b[p][j] = *(const f16x8_t*)(fb + (p * FB + j) * ORTH_BLOCK);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                f16x8_t a[PA];
#pragma unroll
                for (int p = 0; p < PA; ++p) a[p] = *(const f16x8_t*)(fa + (p * FA + i) * ORTH_BLOCK);
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[0][j], a[0], acc[i][j], 0, 0, 0);
                if constexpr (PB == 2) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[1][j], a[0], acc[i][j], 0, 0, 0);
                }
                if constexpr (PA == 2) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[0][j], a[1], acc[i][j], 0, 0, 0);
                }
            }
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
    }

    // A lane has the columns 4 (lane / 16) + 0..3 of row lane % 16 of every fragment.
    const int i = lane & 15, q = lane >> 4;
    const int row0 = (tm * FA + wm * FM) * 16, col0 = (tn * FB + wn * FN) * 16;
#pragma unroll
    for (int m = 0; m < FM; ++m) {
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            const int r = row0 + m * 16, c = col0 + n * 16;  // of the fragment
            f32x4_t v = acc[m][n];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= g.alpha;
            // within the block of 32 columns: 16 rows times (c % 32) / 8 columns of eight
            const int64_t here = ((int64_t)(r >> 4) * (CIN > 0 ? g.cin.blocks : g.c.blocks) + (c >> 5)) * ORTH_BLOCK + (i + 16 * ((c >> 3 & 2) + (q >> 1))) * 16 + (q & 1) * 8;
            if constexpr (CIN > 0) {
                const char* in = g.cin.part[0] + matrix * g.cin.matrix + here;
                const u32x2_t hi = *(const u32x2_t*)in;
                v[0] = fmaf(g.beta, f16_lo(hi[0]), v[0]), v[1] = fmaf(g.beta, f16_hi(hi[0]), v[1]);
                v[2] = fmaf(g.beta, f16_lo(hi[1]), v[2]), v[3] = fmaf(g.beta, f16_hi(hi[1]), v[3]);
                if constexpr (CIN == 2) {
                    const u32x2_t lo = *(const u32x2_t*)(g.cin.part[1] + matrix * g.cin.matrix + here);
                    v[0] = fmaf(g.beta, f16_lo(lo[0]), v[0]), v[1] = fmaf(g.beta, f16_hi(lo[0]), v[1]);
                    v[2] = fmaf(g.beta, f16_lo(lo[1]), v[2]), v[3] = fmaf(g.beta, f16_hi(lo[1]), v[3]);
                }
            }
            if constexpr (OUT == ORTH_SQUARE || OUT == ORTH_BLOCKS) {
                // the transpose's block: 16 columns times (r % 32) / 8 groups of eight rows
                const int64_t there = ((int64_t)(c >> 4) * g.ct.blocks + (r >> 5)) * ORTH_BLOCK + (4 * q + (i & 3) + 16 * ((r >> 3 & 2) + (i >> 3))) * 16 + (i >> 2 & 1) * 8;
                uint32_t w[2] = {pack_f16(v[0], v[1]), pack_f16(v[2], v[3])};
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    if (p == 1) {
                        const uint32_t h0 = w[0], h1 = w[1];
                        w[0] = pack_f16(v[0] - f16_lo(h0), v[1] - f16_hi(h0));
                        w[1] = pack_f16(v[2] - f16_lo(h1), v[3] - f16_hi(h1));
                    }
                    *(u32x2_t*)(g.c.part[p] + matrix * g.c.matrix + here) = u32x2_t{w[0], w[1]};
                    if (!SYM || tm != tn) {
                        uint32_t x = w[0], y = w[1];
                        turn_f16(x, y);
                        *(u32x2_t*)(g.ct.part[p] + matrix * g.ct.matrix + there) = u32x2_t{x, y};
                    }
                }
            } else {
                if (g.tall) turn_f32(v);  // rows and columns change places: 4 of the caller's neighbouring values again
                const int rr = g.tall ? c + 4 * q + (i & 3) : r + i, cc = g.tall ? r + (i & 12) : c + 4 * q;
                const int rows = g.tall ? g.cols : g.rows, cols = g.tall ? g.rows : g.cols;
                if (rr < rows) {
                    const int64_t to = matrix * g.out_matrix + rr * g.out_ld + cc;
                    if (g.vec && cc + 3 < cols) {
                        if constexpr (OUT == ORTH_F32) {
                            *(f32x4_t*)((float*)g.out + to) = v;
                        } else {
                            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                            *(bf16x4_t*)((uint16_t*)g.out + to) = bf16x4_t{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (cc + j >= cols) continue;
                            if constexpr (OUT == ORTH_F32) ((float*)g.out)[to + j] = v[j];
                            else ((__bf16*)g.out)[to + j] = (__bf16)v[j];
                        }
                    }
                }
            }
        }
    }
}

// ---- the way in ----
constexpr int kThreads = 256;

struct OrthIn {
    const void* g;
    int64_t matrix, ld;  // values from one matrix, one row to the next
    int rows, cols;
    double* partials;    // [matrices][parts]
    int parts;
    float eps;
    OrthOperand x, xt;   // G in blocks along its columns, and along its rows
};

template <typename T> static __device__ inline float value_of(const T* p) { return (float)*p; }
template <> __device__ inline float value_of<uint16_t>(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

static __device__ inline double block_sum(double v, double* lds) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
    for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
    return s;
}

// Squares of a matrix, in 64 bits: part blockIdx.x of the rows.
template <typename T> __global__ __launch_bounds__(kThreads) void orth_squares_kernel(OrthIn in) {
    __shared__ double lds[kThreads / 64];
    const T* g = (const T*)in.g + blockIdx.y * in.matrix;
    const int per = (in.rows + in.parts - 1) / in.parts, from = blockIdx.x * per, to = min(from + per, in.rows);
    double s = 0;
    for (int64_t i = threadIdx.x; i < (int64_t)(to - from) * in.cols; i += kThreads) {
        const int64_t r = i / in.cols;
        const double v = value_of(g + (from + r) * in.ld + (i - r * in.cols));
        s = fma(v, v, s);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) in.partials[(int64_t)blockIdx.y * in.parts + blockIdx.x] = s;
}

// 64 x 64 values into blocks of both kinds, in two parts
template <typename T> __global__ __launch_bounds__(kThreads) void orth_blocks_kernel(OrthIn in) {
    __shared__ double lds[kThreads / 64];
    __shared__ float tile[64][65];
    const int matrix = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const T* g = (const T*)in.g + matrix * in.matrix;
    double s = 0;
    for (int i = threadIdx.x; i < in.parts; i += kThreads) s += in.partials[(int64_t)matrix * in.parts + i];
    const double scale = (double)X_SCALE / (sqrt(block_sum(s, lds)) + (double)in.eps);
    for (int i = threadIdx.x; i < 64 * 64; i += kThreads) {
        const int r = i >> 6, c = i & 63;
        tile[r][c] = r0 + r < in.rows && c0 + c < in.cols ? (float)((double)value_of(g + (int64_t)(r0 + r) * in.ld + c0 + c) * scale) : 0.f;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * 512; k += kThreads) {  // 16-byte pieces: 8 blocks of 64 lanes of each kind
        const bool turned = k >= 512;
        const int piece = k & 511, l = piece & 63, br = piece >> 7, bc = piece >> 6 & 1;  // 4 x 2 blocks
        const int row = br * 16 + (l & 15), col = bc * 32 + (l >> 4) * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = turned ? tile[col + j][row] : tile[row][col + j];
        u32x4_t hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            hi[j] = pack_f16(v[2 * j], v[2 * j + 1]);
            lo[j] = pack_f16(v[2 * j] - f16_lo(hi[j]), v[2 * j + 1] - f16_hi(hi[j]));
        }
        const OrthOperand& o = turned ? in.xt : in.x;
        const int R = (turned ? c0 : r0) / 16 + br, C = (turned ? r0 : c0) / 32 + bc;
        const int64_t at = matrix * o.matrix + ((int64_t)R * o.blocks + C) * ORTH_BLOCK + l * 16;
        *(u32x4_t*)(o.part[0] + at) = hi;
        *(u32x4_t*)(o.part[1] + at) = lo;
    }
}

// ---- plan ----
struct Size {
    int n, m;        // of X, padded
    int tile;        // 256 or 128
    int parts;       // of the squares
    int64_t x, s;    // bytes of a plane of X and of S
};

Size size_of_matrix(int rows, int cols) {
    Size z;
    const int n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    z.tile = n > 256 ? 256 : 128;
    z.n = (n + z.tile - 1) / z.tile * z.tile;
    z.m = (m + z.tile - 1) / z.tile * z.tile;
    z.x = (int64_t)z.n * z.m * 2;
    z.s = (int64_t)z.n * z.n * 2;
    const int64_t want = ((int64_t)rows * cols + 16383) / 16384;
    z.parts = (int)(want < 256 ? want : 256);
    if (z.parts > rows) z.parts = rows;
    return z;
}

// X in two parts, X^T in two parts twice (one is read while the next is written), S and P in two parts; the partial sums
int64_t matrix_bytes(const Size& z) { return 6 * z.x + 4 * z.s + 4096; }

template <int PA, int PB, int CIN, int PARTS, int OUT> hipError_t product(const OrthArgs& g, int tile, hipStream_t st) {
    auto run = [&](auto kernel, int bytes, int threads) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        kernel<<<g.tiles * g.matrices, threads, bytes, st>>>(g);
        return hipGetLastError();
    };
    constexpr int PLANES = PA + PB, KS = PLANES == 2 ? 2 : 1, STAGES = PLANES == 2 ? 4 : PLANES == 3 ? 3 : 2;
    if (tile == 256) return run(orth_product_kernel<PA, PB, 2, 4, 8, 4, KS, 2, CIN, PARTS, OUT>, 16 * PLANES * KS * 2 * ORTH_BLOCK, 512);
    return run(orth_product_kernel<PA, PB, 2, 2, 4, 4, 1, STAGES, CIN, PARTS, OUT>, 8 * PLANES * STAGES * ORTH_BLOCK, 256);
}

OrthOperand operand(char*& at, int64_t plane, int parts, int blocks, int matrices) {
    OrthOperand o = {};
    for (int p = 0; p < parts; ++p) {
        o.part[p] = at;
        at += plane * matrices;
    }
    o.matrix = plane;
    o.blocks = blocks;
    return o;
}

template <bool F32> hipError_t steps_of(const OrthTask& t, const Size& z, const OrthIn& in, OrthOperand x, OrthOperand xt, OrthOperand xt2, OrthOperand s,
                                        OrthOperand p, int count, void* out, hipStream_t st) {
    constexpr int PARTS = F32 ? 2 : 1;
    const int nt = z.n / z.tile, mt = z.m / z.tile;
    for (int k = 0; k < t.steps; ++k) {
        const float *abc = t.coefficients + 3 * k, a = abc[0], b = abc[1], c = abc[2];
        OrthArgs g = {};
        g.matrices = count;
        g.mt = g.nt = nt;
        g.tiles = nt * (nt + 1) / 2;
        g.a = g.b = x;
        g.c = g.ct = s;
        g.steps = z.m / 32;
        g.alpha = S_SCALE / (X_SCALE * X_SCALE);
        hipError_t e = product<PARTS, PARTS, 0, 2, ORTH_SQUARE>(g, z.tile, st);
        if (e != hipSuccess) return e;
        g.a = g.b = g.cin = s;
        g.c = g.ct = p;
        g.steps = z.n / 32;
        g.alpha = c * P_SCALE / (S_SCALE * S_SCALE);
        g.beta = b * P_SCALE / S_SCALE;
        e = product<2, 2, 2, PARTS, ORTH_SQUARE>(g, z.tile, st);
        if (e != hipSuccess) return e;
        g.a = p;
        g.b = xt;
        g.cin = g.c = x;
        g.ct = xt2;
        g.mt = nt;
        g.nt = mt;
        g.tiles = nt * mt;
        const bool last = k == t.steps - 1;
        g.alpha = (last ? t.scale / X_SCALE : 1.f) / P_SCALE;
        g.beta = last ? t.scale / X_SCALE * a : a;
        if (!last) {
            e = product<PARTS, 2, 2, 2, ORTH_BLOCKS>(g, z.tile, st);
        } else {
            g.out = out;
            g.out_matrix = t.out_matrix;
            g.out_ld = t.out_ld;
            g.tall = t.rows > t.cols;
            g.rows = g.tall ? t.cols : t.rows;
            g.cols = g.tall ? t.rows : t.cols;
            const int size = F32 ? 4 : 2;
            g.vec = ((uintptr_t)out & (4 * size - 1)) == 0 && t.out_ld % 4 == 0 && (count == 1 || t.out_matrix % 4 == 0);
            e = product<PARTS, 2, 2, 0, F32 ? ORTH_F32 : ORTH_BF16>(g, z.tile, st);
        }
        if (e != hipSuccess) return e;
        const OrthOperand o = xt;
        xt = xt2;
        xt2 = o;
    }
    return hipSuccess;
}

}  // namespace

// A few matrices at a time where the whole stack would take more than this
constexpr int64_t ORTH_WORKSPACE = (int64_t)8 << 30;

size_t orth_workspace(int E, int rows, int cols) {
    const int64_t one = matrix_bytes(size_of_matrix(rows, cols));
    int64_t count = ORTH_WORKSPACE / one;
    if (count > E) count = E;
    return (size_t)((count > 1 ? count : 1) * one);
}

hipError_t launch_orth(const OrthTask& t, void* workspace, hipStream_t st) {
    const Size z = size_of_matrix(t.rows, t.cols);
    const int at_once = (int)(orth_workspace(t.E, t.rows, t.cols) / matrix_bytes(z));
    const bool tall = t.rows > t.cols;
    const int size_in = t.in_f32 ? 4 : 2, size_out = t.out_f32 ? 4 : 2;
    for (int e0 = 0; e0 < t.E; e0 += at_once) {
        const int count = t.E - e0 < at_once ? t.E - e0 : at_once;
        char* at = (char*)workspace;
        const OrthOperand x = operand(at, z.x, 2, z.m / 32, count), xt = operand(at, z.x, 2, z.n / 32, count), xt2 = operand(at, z.x, 2, z.n / 32, count);
        const OrthOperand s = operand(at, z.s, 2, z.n / 32, count), p = operand(at, z.s, 2, z.n / 32, count);
        OrthIn in = {};
        in.g = (const char*)t.g + e0 * t.g_matrix * size_in;
        in.matrix = t.g_matrix;
        in.ld = t.g_ld;
        in.rows = t.rows;
        in.cols = t.cols;
        in.partials = (double*)at;
        in.parts = z.parts;
        in.eps = t.eps;
        in.x = tall ? xt : x;
        in.xt = tall ? x : xt;
        const dim3 blocks((tall ? z.n : z.m) / 64, (tall ? z.m : z.n) / 64, count);
        if (t.in_f32) {
            orth_squares_kernel<float><<<dim3(z.parts, count), kThreads, 0, st>>>(in);
            orth_blocks_kernel<float><<<blocks, kThreads, 0, st>>>(in);
        } else {
            orth_squares_kernel<uint16_t><<<dim3(z.parts, count), kThreads, 0, st>>>(in);
            orth_blocks_kernel<uint16_t><<<blocks, kThreads, 0, st>>>(in);
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        void* out = (char*)t.out + e0 * t.out_matrix * size_out;
        e = t.out_f32 ? steps_of<true>(t, z, in, x, xt, xt2, s, p, count, out, st) : steps_of<false>(t, z, in, x, xt, xt2, s, p, count, out, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
