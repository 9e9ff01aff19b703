// Stacks of matrices brought near the orthogonal matrices next to them by Newton-Schulz steps:
//   X = G / (|G| + eps);  for each step (a, b, c):  S = X X^T,  P = b S + c S S,  X = a X + P X;  out = scale X.
// (tall matrices: the same on the transpose).  Singular vectors stay, and each singular value s goes through a s + b s^3 + c s^5.
//
// Products bound it: of n x m matrices, n <= m, n n m + n n n + 2 n n m operations a step where the two symmetric products are formed on
// and above the diagonal only.  Matrix instructions take 16-bit operands, and what a step rounds is multiplied by the ones behind it (by a
// each, for the small singular values), so operands are kept in one or two parts of fp16 (moe_orth.h), and X always in two.
//   fp32 results: all operands of all products have two parts, 22 bits: no further from the exact ones than those of 32-bit products, but for a few small
// matrices (1e-6 to 1.5e-5 of their norm; 0.2 to 1 times, 1.5 for 100 to 150 rows and steps that raise small values by 8).  Three products of parts for one, so where X is wide two steps are taken at a time through products of squares only.
//   bf16 results: one part in every product; beside it the diagonal of Q = a I + b S + c S S, its largest share, is kept in 32 bits, for X's second part and
// for what its own rounding takes from the first.  Of five usual steps 1e-4 of the norm on the spectra of gradients, 8e-4 on flat ones, below the 1.66e-3 of the
// result's own rounding (1.00 to 1.14 times that in all; without the latter 1.03 to 1.22, and 2.6 for 300 x 400 and the steps of 8; with X in one part steep
// spectra lose 8e-3, with bf16 operands 6e-2).  More steps carry it further (eight 1.06 to 1.43), and steps whose slope is large where singular values come
// to lie: 1.0 to 1.8 for the steps of 8, up to 2.5 after four of them; damped by 1 % they stay within 1.24.
// Measured: 8 matrices of 4096 x 14336 in bf16 30.8 ms (1025 TFLOP/s of the operations above; single products 1070 with X, whose tiles read and write X's
// parts, and 1130 for S), 32 of 7168 x 2048 in fp32 30.6 ms (1145 TFLOP/s of the products of parts), 128 of 768 x 2048 in bf16 4.4 ms.  One-part
// products wait for their operands on the way from the L2s through LDS (without these loads the first case takes two thirds of its time); short
// reductions, as 768, for tiles' beginnings and ends.
#include "moe_orth.h"

#include <math.h>

#include <initializer_list>

namespace {

// X, S and Q = a I + b S + c S S are held times powers of two: in the middle of fp16's range, so that the second parts are seldom subnormal.  These where
// the coefficients allow them, which the usual ones do (singular values below 2 on the way, Q below 16); less where they lead further, down to these
// (singular values of 16, Q of 4094).
constexpr float X_SCALE = 8192.f, S_SCALE = 4096.f, Q_SCALE = 2048.f;
constexpr float X_LEAST = 1024.f, S_LEAST = 64.f, Q_LEAST = 8.f;

// Where |G| is far below eps, X is small, and its parts would be subnormal: it is kept another power of two higher, so that its norm begins in [1/2, 1).
// The steps raise it (all of it by a, as S is next to nothing), so the lift sinks from step to step by what they may have raised it, to nothing.
// The sums that a step forms of X take the lift out again: S = X X^T twice, the next X, but for the lift that it has.
constexpr int LIFT_MOST = 96;
// (by a vector load, which nothing waits for before it is used; a wait for the kernel's arguments would wait for a scalar one too: 2048 x 2048 in bf16 427 and 432 us)
static __device__ inline int fetch_lift(const OrthArgs& g, int matrix) {
    asm("" : "+v"(matrix));
    return g.lift[matrix];
}
static __device__ inline int sunk_lift(int lift, int sunk) { return max(lift - sunk, 0); }
static __device__ inline float unlifted(const OrthArgs& g, int lift) { return ldexpf(1.f, sunk_lift(lift, g.sunk_after) - g.lifts * sunk_lift(lift, g.sunk)); }

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

// The tile t of a matrix: (row, column) of tiles
template <bool SYM> static __device__ inline void place(const OrthArgs& g, int t, int* tm, int* tn) {
    int m, n;
    if constexpr (SYM) {
        place_symmetric(t, g.mt, &m, &n);
    } else {  // bands of 8 tiles
        const int band = t / (8 * g.nt), r = t - band * 8 * g.nt, h = min(8, g.mt - 8 * band);
        n = r / h;
        m = 8 * band + r - n * h;
    }
    *tm = __builtin_amdgcn_readfirstlane(m);
    *tn = __builtin_amdgcn_readfirstlane(n);
}

// The sums of two neighbouring fragments on their way out: a lane has the columns c + 4 q + 0..3 and c + 16 + 4 q + 0..3 of row r + i (i = lane % 16,
// q = lane / 16).  CIN: parts of another matrix that is added beta times; ROWS: each row of each part beta times its number in `own`.
// OUT: a symmetric result in blocks, whose tiles above the diagonal (`both`) are written to both sides; any result in blocks; or its type in
// the caller's rows.  PARTS: of a result in blocks.
// unlift: what takes the lift of X out of the sums.
// In a block a lane's 4 values are half a piece, and lanes of neighbouring q change halves for accesses of 16 bytes.
template <int CIN, bool ROWS, int PARTS, int OUT> static __device__ inline void finish(const OrthArgs& g, float unlift, f32x4_t u, f32x4_t v, int lane, int matrix, int r, int c, bool both) {
    const int i = lane & 15, q = lane >> 4;
    const int64_t here = ((int64_t)(r >> 4) * g.c.blocks + (c >> 5)) * ORTH_BLOCK + orth_piece(i, (q & 1) * 2 + (q >> 1)) * 16;
    u *= g.alpha * unlift;
    v *= g.alpha * unlift;
    if constexpr (CIN > 0) {
        f32x2_t betas = {g.beta * unlift, g.beta * unlift};
        if (ROWS) betas *= *(const f32x2_t*)(g.own + ((int64_t)matrix * g.square + r + i) * 2);
#pragma unroll
        for (int p = 0; p < CIN; ++p) {
            const float beta = betas[p];
            const u32x4_t w = *(const u32x4_t*)(g.cin.part[p] + matrix * g.cin.matrix + here);
            const auto x = __builtin_amdgcn_permlane16_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane16_swap(w[1], w[3], false, false);
            u[0] = fmaf(beta, f16_lo(x[0]), u[0]), u[1] = fmaf(beta, f16_hi(x[0]), u[1]), u[2] = fmaf(beta, f16_lo(y[0]), u[2]), u[3] = fmaf(beta, f16_hi(y[0]), u[3]);
            v[0] = fmaf(beta, f16_lo(x[1]), v[0]), v[1] = fmaf(beta, f16_hi(x[1]), v[1]), v[2] = fmaf(beta, f16_lo(y[1]), v[2]), v[3] = fmaf(beta, f16_hi(y[1]), v[3]);
        }
    }
    if constexpr (OUT == ORTH_SQUARE) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (r == c) u[j] += 4 * q + j == i ? g.diagonal : 0.f;
            if (r == c + 16) v[j] += 4 * q + j == i ? g.diagonal : 0.f;
        }
    }
    if constexpr (OUT == ORTH_SQUARE || OUT == ORTH_BLOCKS) {
        uint32_t parts[2][4];
        split_f16(u[0], u[1], parts[0][0], parts[1][0]), split_f16(u[2], u[3], parts[0][1], parts[1][1]);
        split_f16(v[0], v[1], parts[0][2], parts[1][2]), split_f16(v[2], v[3], parts[0][3], parts[1][3]);
        if constexpr (OUT == ORTH_SQUARE && PARTS == 1) {
            if (g.own != nullptr && (r == c || r == c + 16)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t word = parts[0][(r == c ? 0 : 2) + j / 2];
                    const float x = r == c ? u[j] : v[j], kept = j % 2 == 0 ? f16_lo(word) : f16_hi(word);
                    if (4 * q + j == i) *(f32x2_t*)(g.own + ((int64_t)matrix * g.square + r + i) * 2) = f32x2_t{(x - kept) * g.unscale, x * g.unscale};
                }
            }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const uint32_t(&a)[4] = parts[p];
            char* to = g.c.part[p] + matrix * g.c.matrix;
            const auto x = __builtin_amdgcn_permlane16_swap(a[0], a[2], false, false), y = __builtin_amdgcn_permlane16_swap(a[1], a[3], false, false);
            *(u32x4_t*)(to + here) = u32x4_t{x[0], y[0], x[1], y[1]};
            if (OUT == ORTH_SQUARE && both) {  // the same on the other side, 4 rows of a column a lane
                const int64_t there = ((int64_t)(c >> 4) * g.c.blocks + (r >> 5)) * ORTH_BLOCK + orth_piece(4 * q + (i & 3), (r >> 3 & 2) + (i >> 3)) * 16 + (i >> 2 & 1) * 8;
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    uint32_t s = a[2 * f], t = a[2 * f + 1];
                    turn_f16(s, t, lane);
                    *(u32x2_t*)(to + there + f * (int64_t)g.c.blocks * ORTH_BLOCK) = u32x2_t{s, t};
                }
            }
        }
    } else {
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            f32x4_t x = f == 0 ? u : v;
            const int cf = c + 16 * f;
            if (g.tall) turn_f32(x, lane);  // rows and columns change places: 4 of the caller's neighbouring values again
            const int rr = g.tall ? cf + 4 * q + (i & 3) : r + i, cc = g.tall ? r + (i & 12) : cf + 4 * q;
            const int rows = g.tall ? g.cols : g.rows, cols = g.tall ? g.rows : g.cols;
            if (rr >= rows) continue;
            const int64_t to = matrix * g.out_matrix + rr * g.out_ld + cc;
            if (g.vec && cc + 3 < cols) {
                if constexpr (OUT == ORTH_F32) {
                    *(f32x4_t*)((float*)g.out + to) = x;
                } else {
                    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
                    *(bf16x4_t*)((uint16_t*)g.out + to) = bf16x4_t{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (cc + j >= cols) continue;
                    if constexpr (OUT == ORTH_F32) ((float*)g.out)[to + j] = x[j];
                    else ((__bf16*)g.out)[to + j] = (__bf16)x[j];
                }
            }
        }
    }
}

// PA, PB: parts of A and B.  TB: B lies with the reduction along its rows (otherwise along its columns).  WM x WN wavefronts of FM x FN
// fragments (16 x 16).  A stage is KS blocks of 32 of the reduction, STAGES of them in LDS.  CIN, ROWS, PARTS, OUT: what finish makes of the sums.
template <int PA, int PB, bool TB, int WM, int WN, int FM, int FN, int KS, int STAGES, int CIN, bool ROWS, int PARTS, int OUT>
__global__ __launch_bounds__(WM* WN * 64, 2) void orth_product_kernel(OrthArgs g) {
    constexpr int WAVES = WM * WN, FA = WM * FM, FB = WN * FN, FRAGS = KS * (FA * PA + FB * PB), LOADS = FRAGS / WAVES;
    static_assert(FA % WAVES == 0 && FB == 2 * WAVES, "a load's operand and block row do not depend on the wavefront");
    constexpr bool SYM = OUT == ORTH_SQUARE;
    extern __shared__ __align__(1024) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN, i16 = lane & 15, q16 = lane >> 4;

    // neighbouring tiles on one XCD (workgroup number % 8): one stretch of the list each
    const bool cut = (int)blockIdx.x >= g.whole;
    const int number = blockIdx.x - (cut ? g.whole : 0), total = cut ? (g.tiles * g.matrices - g.whole) * g.splits : g.whole;
    const int xcd = number & 7, each = total >> 3, rest = total & 7;
    int item = xcd * each + min(xcd, rest) + (number >> 3);
    const int64_t slot = item;
    const int splits = cut ? g.splits : 1, split = item % splits;
    item = cut ? g.whole + item / splits : item;
    const int matrix = item / g.tiles;
    int tm, tn;
    place<SYM>(g, item - matrix * g.tiles, &tm, &tn);
    const int lift = SYM && CIN > 0 ? 0 : fetch_lift(g, matrix);  // (needed at the end)

    // A stage's loads: block row i * WAVES + wave of an operand along its columns; of one along its rows block row i, block column wave.
    const uint32_t panel = (uint32_t)g.a.blocks * ORTH_BLOCK, panel_b = (uint32_t)g.b.blocks * ORTH_BLOCK;
    u32x4_t da[PA], db[PB];
#pragma unroll
    for (int p = 0; p < PA; ++p) da[p] = orth_desc(g.a.part[p] + matrix * g.a.matrix + (int64_t)tm * FA * panel, FA * panel);
#pragma unroll
    for (int p = 0; p < PB; ++p) {
        const int64_t at = TB ? (int64_t)tn * (FB / 2) * ORTH_BLOCK : (int64_t)tn * FB * panel_b;
        db[p] = orth_desc(g.b.part[p] + matrix * g.b.matrix + at, TB ? (uint32_t)(g.b.matrix - at) : FB * panel_b);
    }
    constexpr int NA = FA / WAVES, NB = FB / WAVES, PER = PA * NA + PB * NB;  // loads of a block of the reduction
    // (places beside the lane's are scalars: a register a load more, and the longest loop spilled)
    const uint32_t mine = lane * 16, wave_a = wave * panel, wave_b = TB ? wave * ORTH_BLOCK : wave * panel_b;
    const uint32_t base = __builtin_amdgcn_readfirstlane(orth_lds_addr(lds)) + wave * ORTH_BLOCK;
    auto issue_one = [&](auto load, int s, int place) {  // one load of stage s
        constexpr int k = decltype(load)::value / PER, i = decltype(load)::value % PER, ib = i - PA * NA;
        const uint32_t to = base + place * (FRAGS * ORTH_BLOCK), at = (uint32_t)(s * KS + k);
        if constexpr (i < PA * NA) {
            orth_load(to + (KS * (i / NA) * FA + k * FA + i % NA * WAVES) * ORTH_BLOCK, mine, da[i / NA], at * ORTH_BLOCK + wave_a + i % NA * WAVES * panel);
        } else {
            const uint32_t rows = TB ? (2 * at + ib % NB) * panel_b : at * ORTH_BLOCK + ib % NB * WAVES * panel_b;
            orth_load(to + (KS * (PA * FA + ib / NB * FB) + k * FB + ib % NB * WAVES) * ORTH_BLOCK, mine, db[ib / NB], rows + wave_b);
        }
    };
    auto issue = [&](int s, int place) { orth_repeat<LOADS>([&](auto load) { issue_one(load, s, place); }); };

    f32x4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    f16x8_t a[KS][PA][FM], b[KS][PB][FN];
    const int stages = g.steps / KS, first = (int)((int64_t)stages * split / splits), end = (int)((int64_t)stages * (split + 1) / splits);
    const int at_row = orth_piece(i16, q16) * 16;
    // of the transposing read: lane i of 16 asks for 4 columns of row 8 (q % 2) + i / 4 and is given column i of 4 rows; the next 4 rows lie where
    // the exclusive or with 12 of the rows puts them
    const int t_row = 8 * (q16 & 1) + (i16 >> 2), t_g = (i16 & 3) >> 1;
    const int at_turn = orth_piece(t_row, t_g) * 16 + (i16 & 1) * 8, at_next = orth_piece(t_row + 4, t_g) * 16 + (i16 & 1) * 8;
    auto read = [&](int place) {
        const char* at = lds + place * (FRAGS * ORTH_BLOCK);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int p = 0; p < PB; ++p)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const char* block = at + (KS * (PA * FA + p * FB) + k * FB) * ORTH_BLOCK;
                    if constexpr (TB) {
                        typedef short s16x4_t __attribute__((ext_vector_type(4)));
                        typedef short s16x8_t __attribute__((ext_vector_type(8)));
                        typedef __attribute__((address_space(3))) s16x4_t lds4;
                        block += ((q16 >> 1) * WAVES + (wn * FN + j) / 2) * ORTH_BLOCK + j % 2 * 512;
                        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_turn)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_next));
                        b[k][p][j] = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
                        b[k][p][j] = *(const f16x8_t*)(block + (wn * FN + j) * ORTH_BLOCK + at_row);
                    }
                }
#pragma unroll
            for (int p = 0; p < PA; ++p)
#pragma unroll
                for (int i = 0; i < FM; ++i) a[k][p][i] = *(const f16x8_t*)(at + (KS * p * FA + k * FA + wm * FM + i) * ORTH_BLOCK + at_row);
        }
    };
    constexpr int PAIRS = PA + PB - 1, LINES = KS * PAIRS * FM;  // rows of fragments that a stage's products come in
    auto multiply = [&](auto&& beside) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        orth_repeat<LINES>([&](auto row) {
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

    if constexpr (WAVES == 8) {
        // Two groups of four wavefronts, one of each on every SIMD, take turns: while one group multiplies, the other reads its next
        // fragments, so the matrix cores always have a wavefront whose operands are there.  In turn 2 s the first group reads stage s (and
        // asks for stage s + 1, into the place that the second group left in the turn before), in 2 s + 1 the second; a stage has two turns to
        // arrive.
        static_assert(STAGES == 2, "");
        issue(first, first & 1);
        orth_wait<0>();
        orth_barrier();
        const bool ahead = wave < 4;
        if (!ahead) {
            if (first + 1 < end) issue(first + 1, (first + 1) & 1);
            orth_barrier();
        }
        for (int s = first; s < end; ++s) {  // one loop for both groups: two copies of it cost registers
            read(s & 1);
            if (ahead) {
                if (s + 1 < end) issue(s + 1, (s + 1) & 1);
            } else {
                orth_wait<0>();
            }
            orth_barrier();
            const bool more = !ahead && s + 2 < end;
            multiply([&](auto row) {  // the second group's loads among its products
                constexpr int r = decltype(row)::value;
                if constexpr (r * LOADS % LINES < LOADS && r * LOADS / LINES < LOADS) {
                    if (more) issue_one(OrthInt<r * LOADS / LINES>{}, s + 2, s & 1);
                }
            });
            if (ahead) orth_wait<0>();
            orth_barrier();
        }
        if (ahead) orth_barrier();
    } else {
        orth_repeat<STAGES - 1>([&](auto s) {
            if (first + decltype(s)::value < end) issue(first + decltype(s)::value, decltype(s)::value);
        });
        int place = 0;
        for (int s = first; s < end; ++s) {
            // this stage has arrived; the last ones have fewer behind them and wait for all
            if (s + STAGES - 1 <= end) orth_wait<(STAGES - 2) * LOADS>();
            else orth_wait<0>();
            orth_barrier();  // of every wavefront's; and all are done with the stage before
            if (s + STAGES - 1 < end) issue(s + STAGES - 1, place == 0 ? STAGES - 1 : place - 1);
            read(place);
            multiply([](auto) {});
            place = place == STAGES - 1 ? 0 : place + 1;
        }
    }

    int out_lane = lane;
    asm volatile("" : "+v"(out_lane));  // the compiler would form the results' places before the loop and spill them
    if (cut) {
        f32x4_t* part = (f32x4_t*)g.part + slot * (FA * FB * 64) + out_lane;
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) part[((wm * FM + m) * FB + wn * FN + n) * 64] = acc[m][n];
        return;
    }
    const float unlift = SYM && CIN > 0 ? 1.f : unlifted(g, lift);
    const int row0 = (tm * FA + wm * FM) * 16, col0 = (tn * FB + wn * FN) * 16;
#pragma unroll
    for (int m = 0; m < FM; ++m) {
        if (m % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < FN; n += 2) finish<CIN, ROWS, PARTS, OUT>(g, unlift, acc[m][n], acc[m][n + 1], out_lane, matrix, row0 + m * 16, col0 + n * 16, tm != tn);
    }
}

// The ranges' sums added in their order, a wavefront two fragments; FA x FB fragments a tile
template <int FA, int FB, int CIN, bool ROWS, int PARTS, int OUT> __global__ __launch_bounds__(256) void orth_sums_kernel(OrthArgs g) {
    const int64_t pair = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), item = pair / (FA * FB / 2);
    const int f = (int)(pair - item * (FA * FB / 2)) * 2, tile = g.whole + (int)item, matrix = tile / g.tiles, lane = threadIdx.x & 63;
    int tm, tn;
    place<OUT == ORTH_SQUARE>(g, tile - matrix * g.tiles, &tm, &tn);
    const int lift = OUT == ORTH_SQUARE && CIN > 0 ? 0 : fetch_lift(g, matrix);
    const f32x4_t* part = (const f32x4_t*)g.part + (item * g.splits * (FA * FB) + f) * 64 + lane;
    f32x4_t u = {0.f, 0.f, 0.f, 0.f}, v = u;
#pragma unroll 4
    for (int s = 0; s < g.splits; ++s) {
        u += part[(int64_t)s * (FA * FB * 64)];
        v += part[(int64_t)s * (FA * FB * 64) + 64];
    }
    finish<CIN, ROWS, PARTS, OUT>(g, OUT == ORTH_SQUARE && CIN > 0 ? 1.f : unlifted(g, lift), u, v, lane, matrix, (tm * FA + f / FB) * 16, (tn * FB + f % FB) * 16, tm != tn);
}

// ... into the first range's place, where one workgroup alone would be long at it: 4 of F fragments a workgroup
__global__ __launch_bounds__(256) void orth_fold_kernel(float* part, int splits, int F) {
    f32x4_t* p = (f32x4_t*)part + (int64_t)blockIdx.y * splits * (F * 64) + (blockIdx.x * 4 + (threadIdx.x >> 6)) * 64 + (threadIdx.x & 63);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) v += p[(int64_t)s * (F * 64)];
    *p = v;
}

// ---- between S and the next product with X, for matrices of up to 128 rows ----
// Of two steps' Q = a I + b S + c S S the product from S's ranges.  One workgroup of NF wavefronts a matrix, everything in LDS: two matrices
// of 16 NF rows in two parts, in blocks.  A wavefront has 2 x NF / 2 fragments.  Up to 64 rows
// all four products of the parts are formed: the smallest matrices have few values to average over (4 x 16 x 400 in fp32: 1.5 times the error of 32-bit products with
// three, 1.2 to 1.3 with four; 8 x 128 x 256: 1.1 and 1.05, but 80 us and 85).
// One loop over the products, each with a loop over the reduction, and no branches in them: the code is run from end to end once or a few times, and
// latencies are half of what it takes (8 matrices of 128 rows, two steps: 19 us, 7 of them the products' own; unrolled with all its products 54; only the
// columns from the diagonal on, half the products, but branches, 28).
template <int NF> __global__ __launch_bounds__(NF * 64) void orth_chain_kernel(OrthArgs g, int apart, int splits, OrthPair pair) {
    extern __shared__ __align__(1024) char lds[];
    constexpr int KB = NF / 2, FN = NF / 2, PLANE = NF * KB * ORTH_BLOCK;
    char *s = lds, *q = lds + 2 * PLANE;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.x;
    const int row0 = wave >> 1 << 1, col0 = (wave & 1) * FN, i = lane & 15, q4 = lane >> 4;
    const int at_row = orth_piece(i, q4) * 16;
    f32x4_t v[2][FN];
    auto each = [&](auto&& f) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) f(m, n);
    };
    // a lane's 4 values of a fragment: columns 16 n + 4 (lane / 16) + 0..3 of row 16 m + lane % 16
    auto at = [&](int m, int n, int blocks) { return ((row0 + m) * blocks + ((col0 + n) >> 1)) * ORTH_BLOCK + orth_piece(i, ((col0 + n) & 1) * 2 + (q4 >> 1)) * 16 + (q4 & 1) * 8; };
    auto put = [&](char* to, int64_t plane, int blocks) {
        each([&](int m, int n) {
            const f32x4_t& x = v[m][n];
            uint32_t hi[2], lo[2];
            split_f16(x[0], x[1], hi[0], lo[0]), split_f16(x[2], x[3], hi[1], lo[1]);
            *(u32x2_t*)(to + at(m, n, blocks)) = u32x2_t{hi[0], hi[1]};
            *(u32x2_t*)(to + plane + at(m, n, blocks)) = u32x2_t{lo[0], lo[1]};
        });
    };

    const int lift = fetch_lift(g, matrix);
    const f32x4_t* part = (const f32x4_t*)g.part + (int64_t)matrix * apart * (NF * NF * 64) + lane;  // (apart: ranges between matrices)
    each([&](int m, int n) { v[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
#pragma unroll 4
    for (int r = 0; r < splits; ++r) each([&](int m, int n) { v[m][n] += part[(r * NF * NF + (row0 + m) * NF + col0 + n) * 64]; });
    const float from = ldexpf(pair.from, -2 * sunk_lift(lift, g.sunk));
    each([&](int m, int n) { v[m][n] *= from; });
    put(s, PLANE, KB);
    __syncthreads();
    constexpr int last = 4;  // of the products
#pragma unroll 1
    for (int op = 0; op <= last; ++op) {
        const bool sum = op == 0 || op == 3;  // of s: a I + b s + c s s; the others: q s (1), s q (2, 4)
        const char *x = op == 1 ? q : s, *y = sum || op == 1 ? s : q;
        each([&](int m, int n) { v[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
        f16x8_t a[2][2][2], b[2][2][FN];  // the next block's are read while this one's are multiplied
        auto read = [&](int k) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
#pragma unroll
                for (int m = 0; m < 2; ++m) a[k & 1][p][m] = *(const f16x8_t*)(x + p * PLANE + ((row0 + m) * KB + k) * ORTH_BLOCK + at_row);
#pragma unroll
                for (int n = 0; n < FN; ++n) b[k & 1][p][n] = *(const f16x8_t*)(y + p * PLANE + ((col0 + n) * KB + k) * ORTH_BLOCK + at_row);
            }
        };
        read(0);
        orth_repeat<KB>([&](auto block) {
            constexpr int k = decltype(block)::value;
            if constexpr (k + 1 < KB) read(k + 1);
            __builtin_amdgcn_sched_barrier(0);
            orth_repeat<NF == 8 ? 3 : 4>([&](auto parts) {
                constexpr int p = decltype(parts)::value >> 1, r = decltype(parts)::value & 1;
                each([&](int m, int n) { v[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[k & 1][r][n], a[k & 1][p][m], v[m][n], 0, 0, 0); });
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        const float* abc = pair.abc[op == 0 ? 0 : 1];
        const float scale = sum ? abc[2] : op == last ? pair.joint : pair.through;
        each([&](int m, int n) { v[m][n] *= scale; });
        if (sum) {
            const float ca = abc[0], cb = abc[1];
            each([&](int m, int n) {
                const u32x2_t hi = *(const u32x2_t*)(s + at(m, n, KB)), lo = *(const u32x2_t*)(s + PLANE + at(m, n, KB));
#pragma unroll
                for (int j = 0; j < 4; ++j) v[m][n][j] = fmaf(cb, j & 1 ? f16_hi(hi[j >> 1]) + f16_hi(lo[j >> 1]) : f16_lo(hi[j >> 1]) + f16_lo(lo[j >> 1]), v[m][n][j]);
                if (row0 + m == col0 + n) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[m][n][j] += 4 * q4 + j == i ? ca : 0.f;
                }
            });
        }
        __syncthreads();
        // op 1 and 2: s = q s q = (q x) (q x)^T
        if (op == last) put(g.c.part[0] + matrix * g.c.matrix, g.c.part[1] - g.c.part[0], g.c.blocks);
        else put(op == 0 ? q : s, PLANE, KB);
        __syncthreads();
    }
}

// Two neighbouring fragments' values as the pieces of a block that a lane stores, in two parts
static __device__ inline void pieces_of(const f32x4_t& u, const f32x4_t& v, u32x4_t (&piece)[2]) {
    uint32_t parts[2][4];
    split_f16(u[0], u[1], parts[0][0], parts[1][0]), split_f16(u[2], u[3], parts[0][1], parts[1][1]);
    split_f16(v[0], v[1], parts[0][2], parts[1][2]), split_f16(v[2], v[3], parts[0][3], parts[1][3]);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint32_t(&a)[4] = parts[p];
        const auto x = __builtin_amdgcn_permlane16_swap(a[0], a[2], false, false), y = __builtin_amdgcn_permlane16_swap(a[1], a[3], false, false);
        piece[p] = u32x4_t{x[0], y[0], x[1], y[1]};
    }
}

// Q = a I + b S + c S S in LDS, in two parts, in blocks, from S's ranges, by four wavefronts: each workgroup that multiplies with Q forms it by itself,
// which costs less than a launch in between.  NF / 4 rows of fragments a wavefront (one, of fewer wavefronts, where there are two).
template <int NF> static __device__ inline void orth_q(const OrthArgs& g, char* s, int matrix, int lift) {
    constexpr int KB = NF / 2, PLANE = NF * KB * ORTH_BLOCK, FM = NF == 8 ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q4 = lane >> 4;
    const bool on = wave * FM < NF;
    const int row0 = on ? wave * FM : 0, at_row = orth_piece(i, q4) * 16;
    f32x4_t v[FM][NF];
    auto each = [&](auto&& f) {
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < NF; ++n) f(m, n);
    };
    auto at = [&](int m, int n) { return ((row0 + m) * KB + (n >> 1)) * ORTH_BLOCK + orth_piece(i, (n & 1) * 2 + (q4 >> 1)) * 16 + (q4 & 1) * 8; };
    auto put = [&] {
        each([&](int m, int n) {
            const f32x4_t& x = v[m][n];
            uint32_t hi[2], lo[2];
            split_f16(x[0], x[1], hi[0], lo[0]), split_f16(x[2], x[3], hi[1], lo[1]);
            *(u32x2_t*)(s + at(m, n)) = u32x2_t{hi[0], hi[1]};
            *(u32x2_t*)(s + PLANE + at(m, n)) = u32x2_t{lo[0], lo[1]};
        });
    };
    const f32x4_t* part = (const f32x4_t*)g.sums + (int64_t)matrix * g.apart * (NF * NF * 64) + lane;
    each([&](int m, int n) { v[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
#pragma unroll 2
    for (int r = 0; r < g.ranges; ++r) each([&](int m, int n) { v[m][n] += part[(r * NF * NF + (row0 + m) * NF + n) * 64]; });
    const float from = ldexpf(g.from, -2 * sunk_lift(lift, g.sunk));
    each([&](int m, int n) { v[m][n] *= from; });
    if (on) put();
    __syncthreads();
    each([&](int m, int n) { v[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f}; });
#pragma unroll
    for (int k = 0; k < KB; ++k) {
        f16x8_t a[2][FM], b[2][NF];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int m = 0; m < FM; ++m) a[p][m] = *(const f16x8_t*)(s + p * PLANE + ((row0 + m) * KB + k) * ORTH_BLOCK + at_row);
#pragma unroll
            for (int n = 0; n < NF; ++n) b[p][n] = *(const f16x8_t*)(s + p * PLANE + (n * KB + k) * ORTH_BLOCK + at_row);
        }
        orth_repeat<NF == 8 ? 3 : 4>([&](auto parts) {
            constexpr int p = decltype(parts)::value >> 1, r = decltype(parts)::value & 1;
            each([&](int m, int n) { v[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[r][n], a[p][m], v[m][n], 0, 0, 0); });
        });
    }
    const float scale = g.abc[2], ca = g.abc[0], cb = g.abc[1];
    each([&](int m, int n) {
        const u32x2_t hi = *(const u32x2_t*)(s + at(m, n)), lo = *(const u32x2_t*)(s + PLANE + at(m, n));
#pragma unroll
        for (int j = 0; j < 4; ++j) v[m][n][j] = fmaf(cb, j & 1 ? f16_hi(hi[j >> 1]) + f16_hi(lo[j >> 1]) : f16_lo(hi[j >> 1]) + f16_lo(lo[j >> 1]), v[m][n][j] * scale);
        if (row0 + m == n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[m][n][j] += 4 * q4 + j == i ? ca : 0.f;
        }
    });
    __syncthreads();
    if (on) put();
    __syncthreads();
}

// ---- matrices of up to 64 rows ----
// A wavefront takes 32 columns of X at a time, all its rows (16 NF): they are few enough that Q X and the new S = X X^T of these columns are formed
// one after the other, so X is read and written once a step and memory, or for small stacks the launches, bound it (128 x 8004 x 17 in fp32: 382 us, by
// tiles and products of their own 1310; 24 x 83: 27, of eight launches).  MODE 0: S of X as it is;
// 1: X = Q X and its S; 2: X = Q X to the caller.  OWN: Q is formed here, from the sums that the launch before has left.
// The results' lanes have the columns 4 q + 0..3 and 16 + 4 q + 0..3 of row i; after the change of halves that the stores want, lane (i, q) has 8
// neighbouring columns of row i, in another order of q than an operand's lanes.  S sums over the columns, so any order will do that both of
// its operands have: the results are operands as they are.
template <int NF, int MODE, int OUT, bool OWN> __global__ __launch_bounds__(256, 2) void orth_thin_kernel(OrthArgs g) {
    constexpr int KB = NF / 2;
    extern __shared__ __align__(1024) char lds[];  // a wavefront's blocks, NF of each part; then the wavefronts' S
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.y, i16 = lane & 15, q16 = lane >> 4;
    const int at_row = orth_piece(i16, q16) * 16;
    const int t_row = 8 * (q16 & 1) + (i16 >> 2), t_g = (i16 & 3) >> 1;
    const int at_turn = orth_piece(t_row, t_g) * 16 + (i16 & 1) * 8, at_next = orth_piece(t_row + 4, t_g) * 16 + (i16 & 1) * 8;
    char* mine = lds + wave * (2 * NF * ORTH_BLOCK);
    const uint32_t to = __builtin_amdgcn_readfirstlane(orth_lds_addr(lds)) + wave * (2 * NF * ORTH_BLOCK);
    const uint32_t line = (uint32_t)g.b.blocks * ORTH_BLOCK;
    u32x4_t desc[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) desc[p] = orth_desc(g.b.part[p] + matrix * g.b.matrix, (uint32_t)g.b.matrix);
    f16x8_t q[2][NF][KB];
    const int lift = MODE > 0 ? fetch_lift(g, matrix) : 0;
    if constexpr (MODE > 0) {
        char* own = lds + 4 * (NF * NF > 2 * NF ? NF * NF : 2 * NF) * ORTH_BLOCK;
        if constexpr (OWN) orth_q<NF>(g, own, matrix, lift);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int m = 0; m < NF; ++m)
#pragma unroll
                for (int k = 0; k < KB; ++k)
                    q[p][m][k] = OWN ? *(const f16x8_t*)(own + (p * NF * KB + m * KB + k) * ORTH_BLOCK + at_row)
                                     : *(const f16x8_t*)(g.a.part[p] + matrix * g.a.matrix + (m * g.a.blocks + k) * ORTH_BLOCK + at_row);
    }
    const float unlift = MODE > 0 ? unlifted(g, lift) : 1.f;
    f32x4_t s[NF][NF];
#pragma unroll
    for (int m = 0; m < NF; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n) s[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int c = blockIdx.x * 4 + wave; c < g.steps; c += gridDim.x * 4) {
        f16x8_t x[2][NF];  // rows of the new X: what S is of
        if constexpr (MODE == 0) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int m = 0; m < NF; ++m) x[p][m] = *(const f16x8_t*)(g.b.part[p] + matrix * g.b.matrix + (int64_t)m * line + c * ORTH_BLOCK + at_row);
        } else {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the columns before have been read)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int m = 0; m < NF; ++m) orth_load(to + (p * NF + m) * ORTH_BLOCK, lane * 16, desc[p], m * line + c * ORTH_BLOCK);
            orth_wait<0>();
            f32x4_t v[NF][2];
#pragma unroll
            for (int m = 0; m < NF; ++m) v[m][0] = v[m][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                f16x8_t b[2][2];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        typedef short s16x4_t __attribute__((ext_vector_type(4)));
                        typedef __attribute__((address_space(3))) s16x4_t lds4;
                        const char* block = mine + (p * NF + 2 * k + (q16 >> 1)) * ORTH_BLOCK + j * 512;
                        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_turn)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_next));
                        b[p][j] = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                orth_repeat<4>([&](auto pair) {
                    constexpr int p = decltype(pair)::value >> 1, r = decltype(pair)::value & 1;
#pragma unroll
                    for (int m = 0; m < NF; ++m)
#pragma unroll
                        for (int j = 0; j < 2; ++j) v[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[r][j], q[p][m][k], v[m][j], 0, 0, 0);
                });
            }
#pragma unroll
            for (int m = 0; m < NF; ++m) {
                if constexpr (MODE == 2) {
                    finish<0, false, 0, OUT>(g, unlift, v[m][0], v[m][1], lane, matrix, m * 16, c * 32, false);
                } else {
                    u32x4_t piece[2];
                    pieces_of(v[m][0] * (g.alpha * unlift), v[m][1] * (g.alpha * unlift), piece);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        x[p][m] = __builtin_bit_cast(f16x8_t, piece[p]);
                        *(u32x4_t*)(g.c.part[p] + matrix * g.c.matrix + (int64_t)m * line + c * ORTH_BLOCK + orth_piece(i16, (q16 & 1) * 2 + (q16 >> 1)) * 16) = piece[p];
                    }
                }
            }
        }
        if constexpr (MODE < 2) {
            orth_repeat<4>([&](auto pair) {
                constexpr int p = decltype(pair)::value >> 1, r = decltype(pair)::value & 1;
#pragma unroll
                for (int m = 0; m < NF; ++m)
#pragma unroll
                    for (int n = 0; n < NF; ++n) s[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[r][n], x[p][m], s[m][n], 0, 0, 0);
            });
        }
    }
    if constexpr (MODE < 2) {  // the four wavefronts' sums, in their order
        __syncthreads();
        f32x4_t* all = (f32x4_t*)lds;
#pragma unroll
        for (int m = 0; m < NF; ++m)
#pragma unroll
            for (int n = 0; n < NF; ++n) all[(wave * NF * NF + m * NF + n) * 64 + lane] = s[m][n];
        __syncthreads();
        f32x4_t* part = (f32x4_t*)g.part + ((int64_t)matrix * gridDim.x + blockIdx.x) * (NF * NF * 64);
        for (int i = threadIdx.x; i < NF * NF * 64; i += 256) part[i] = all[i] + all[i + NF * NF * 64] + all[i + 2 * NF * NF * 64] + all[i + 3 * NF * NF * 64];
    }
}

// ---- matrices of 65 to 128 rows ----
// The same by four wavefronts together, 32 rows each: X's blocks and the new X's pieces go through LDS to all of them, and each keeps its rows of Q
// and of S.  The next columns are asked for while these are multiplied.  (100 x 2000 in fp32: 81 us, by tiles 133; 128 x 14336 in bf16 119 and 174.)
template <int MODE, int OUT, bool OWN> __global__ __launch_bounds__(256, OWN ? 1 : 2) void orth_rows_kernel(OrthArgs g) {
    constexpr int NF = 8, KB = 4, FM = 2, STAGE = 2 * NF * ORTH_BLOCK;
    extern __shared__ __align__(1024) char lds[];  // two stages of X's blocks [part][row], the new X's [part][row]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), matrix = blockIdx.y, i16 = lane & 15, q16 = lane >> 4;
    const int at_row = orth_piece(i16, q16) * 16;
    const int t_row = 8 * (q16 & 1) + (i16 >> 2), t_g = (i16 & 3) >> 1;
    const int at_turn = orth_piece(t_row, t_g) * 16 + (i16 & 1) * 8, at_next = orth_piece(t_row + 4, t_g) * 16 + (i16 & 1) * 8;
    const uint32_t to = __builtin_amdgcn_readfirstlane(orth_lds_addr(lds)), line = (uint32_t)g.b.blocks * ORTH_BLOCK;
    u32x4_t desc[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) desc[p] = orth_desc(g.b.part[p] + matrix * g.b.matrix, (uint32_t)g.b.matrix);
    auto issue = [&](int c, int stage) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int m = 0; m < 2; ++m) orth_load(to + stage * STAGE + (p * NF + m * 4 + wave) * ORTH_BLOCK, lane * 16, desc[p], (m * 4 + wave) * line + c * ORTH_BLOCK);
    };
    char* fresh = lds + 2 * STAGE;
    int stage = 0;
    if (MODE > 0 && (int)blockIdx.x < g.steps) issue(blockIdx.x, 0);
    f16x8_t q[2][FM][KB];
    const int lift = MODE > 0 ? fetch_lift(g, matrix) : 0;
    if constexpr (MODE > 0) {
        char* own = lds + 3 * STAGE;
        if constexpr (OWN) orth_q<NF>(g, own, matrix, lift);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int k = 0; k < KB; ++k)
                    q[p][m][k] = OWN ? *(const f16x8_t*)(own + (p * NF * KB + (wave * FM + m) * KB + k) * ORTH_BLOCK + at_row)
                                     : *(const f16x8_t*)(g.a.part[p] + matrix * g.a.matrix + ((wave * FM + m) * g.a.blocks + k) * ORTH_BLOCK + at_row);
    }
    const float unlift = MODE > 0 ? unlifted(g, lift) : 1.f;
    f32x4_t s[FM][NF];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n) s[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int c = blockIdx.x; c < g.steps; c += gridDim.x) {
        f16x8_t x[2][NF];
        if constexpr (MODE == 0) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int m = 0; m < NF; ++m) x[p][m] = *(const f16x8_t*)(g.b.part[p] + matrix * g.b.matrix + (int64_t)m * line + c * ORTH_BLOCK + at_row);
        } else {
            orth_wait<0>();
            orth_barrier();  // of every wavefront's; and all are done with the columns before
            if (c + (int)gridDim.x < g.steps) issue(c + gridDim.x, stage ^ 1);
            f32x4_t v[FM][2];
#pragma unroll
            for (int m = 0; m < FM; ++m) v[m][0] = v[m][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                f16x8_t b[2][2];
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        typedef short s16x4_t __attribute__((ext_vector_type(4)));
                        typedef __attribute__((address_space(3))) s16x4_t lds4;
                        const char* block = lds + stage * STAGE + (p * NF + 2 * k + (q16 >> 1)) * ORTH_BLOCK + j * 512;
                        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_turn)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(block + at_next));
                        b[p][j] = __builtin_bit_cast(f16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                orth_repeat<3>([&](auto pair) {
                    constexpr int p = decltype(pair)::value >> 1, r = decltype(pair)::value & 1;
#pragma unroll
                    for (int m = 0; m < FM; ++m)
#pragma unroll
                        for (int j = 0; j < 2; ++j) v[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[r][j], q[p][m][k], v[m][j], 0, 0, 0);
                });
            }
            stage ^= 1;
#pragma unroll
            for (int m = 0; m < FM; ++m) {
                const int row = wave * FM + m;
                if constexpr (MODE == 2) {
                    finish<0, false, 0, OUT>(g, unlift, v[m][0], v[m][1], lane, matrix, row * 16, c * 32, false);
                } else {
                    u32x4_t piece[2];
                    pieces_of(v[m][0] * (g.alpha * unlift), v[m][1] * (g.alpha * unlift), piece);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        *(u32x4_t*)(g.c.part[p] + matrix * g.c.matrix + (int64_t)row * line + c * ORTH_BLOCK + orth_piece(i16, (q16 & 1) * 2 + (q16 >> 1)) * 16) = piece[p];
                        *(u32x4_t*)(fresh + (p * NF + row) * ORTH_BLOCK + lane * 16) = piece[p];
                    }
                }
            }
            if constexpr (MODE == 1) {
                orth_barrier();
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int m = 0; m < NF; ++m) x[p][m] = *(const f16x8_t*)(fresh + (p * NF + m) * ORTH_BLOCK + lane * 16);
            }
        }
        if constexpr (MODE < 2) {
            f16x8_t own[2][FM];  // this wavefront's rows of x
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int m = 0; m < FM; ++m) {
                    own[p][m] = x[p][m];
#pragma unroll
                    for (int w = 1; w < 4; ++w) own[p][m] = wave == w ? x[p][w * FM + m] : own[p][m];
                }
            orth_repeat<3>([&](auto pair) {
                constexpr int p = decltype(pair)::value >> 1, r = decltype(pair)::value & 1;
#pragma unroll
                for (int m = 0; m < FM; ++m)
#pragma unroll
                    for (int n = 0; n < NF; ++n) s[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[r][n], own[p][m], s[m][n], 0, 0, 0);
            });
        }
    }
    if constexpr (MODE < 2) {
        f32x4_t* part = (f32x4_t*)g.part + ((int64_t)matrix * gridDim.x + blockIdx.x) * (NF * NF * 64) + lane;
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < NF; ++n) part[((wave * FM + m) * NF + n) * 64] = s[m][n];
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
    int tall;            // G^T is what is put into blocks
    int vec;             // rows begin at multiples of 16 bytes
    int* lift;           // [matrices], for the steps
    int block_rows;      // of x
    OrthOperand x;
};

template <typename T> static __device__ inline float value_of(const T* p) { return (float)*p; }
template <> __device__ inline float value_of<uint16_t>(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

// 16 bytes of values
template <typename T> struct Words;
template <> struct Words<float> {
    static constexpr int N = 4;
    static __device__ inline void open(const u32x4_t& w, float* v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
    }
};
template <> struct Words<uint16_t> {
    static constexpr int N = 8;
    static __device__ inline void open(const u32x4_t& w, float* v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
};

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
    constexpr int N = Words<T>::N;
    const int per = (in.rows + in.parts - 1) / in.parts, from = blockIdx.x * per, to = max(min(from + per, in.rows), from);
    const T* g = (const T*)in.g + blockIdx.y * in.matrix + from * in.ld;
    double s = 0;
    const uint32_t words = in.vec ? in.cols / N : 0, rest = in.cols - words * N, total = (to - from) * words;
    uint32_t i = threadIdx.x;
    auto word = [&](uint32_t k) {
        const uint32_t r = k / words;
        return *(const u32x4_t*)(g + r * in.ld + (k - r * words) * N);
    };
    auto add = [&](const u32x4_t& w) {
        float v[N];
        Words<T>::open(w, v);
#pragma unroll
        for (int j = 0; j < N; ++j) s = fma((double)v[j], (double)v[j], s);
    };
    if (words > 0) {
        for (; i + 3 * kThreads < total; i += 4 * kThreads) {  // four words on their way
            u32x4_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = word(i + k * kThreads);
#pragma unroll
            for (int k = 0; k < 4; ++k) add(w[k]);
        }
        for (; i < total; i += kThreads) add(word(i));
    }
    if (rest > 0) {
        for (uint32_t k = threadIdx.x; k < (to - from) * rest; k += kThreads) {
            const uint32_t r = k / rest;
            const double v = value_of(g + r * in.ld + words * N + (k - r * rest));
            s = fma(v, v, s);
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) in.partials[(int64_t)blockIdx.y * in.parts + blockIdx.x] = s;
}

// 64 x 64 values into blocks, in two parts
template <typename T> __global__ __launch_bounds__(kThreads) void orth_blocks_kernel(OrthIn in) {
    __shared__ double lds[kThreads / 64];
    __shared__ float tile[64][65];
    constexpr int N = Words<T>::N;
    const int matrix = blockIdx.z, r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    const T* g = (const T*)in.g + matrix * in.matrix;
    const bool whole = in.vec && c0 + 64 <= in.cols;  // 16 values of a row a lane
    const int row = threadIdx.x >> 2, col = (threadIdx.x & 3) * 16;
    u32x4_t w[16 / N] = {};
    if (whole && r0 + row < in.rows) {
#pragma unroll
        for (int k = 0; k < 16 / N; ++k) w[k] = *(const u32x4_t*)(g + (int64_t)(r0 + row) * in.ld + c0 + col + k * N);
    }
    double s = 0;
    for (int i = threadIdx.x; i < in.parts; i += kThreads) s += in.partials[(int64_t)matrix * in.parts + i];
    const double norm = sqrt(block_sum(s, lds)), least = norm + (double)in.eps;
    double scale = (double)X_SCALE / least;
    int lift = 0;
    if (norm > 0 && norm < (double)in.eps) {
        (void)frexp(norm / least, &lift);  // (that is below 2^lift)
        lift = min(-lift, LIFT_MOST);
        scale = ldexp(scale, lift);
    }
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) in.lift[matrix] = lift;
    if (whole) {
        const bool live = r0 + row < in.rows;
#pragma unroll
        for (int k = 0; k < 16 / N; ++k) {
            float v[N];
            Words<T>::open(w[k], v);
#pragma unroll
            for (int j = 0; j < N; ++j) tile[row][col + k * N + j] = live ? (float)((double)v[j] * scale) : 0.f;
        }
    } else {
        for (int i = threadIdx.x; i < 64 * 64; i += kThreads) {
            const int r = i >> 6, c = i & 63;
            tile[r][c] = r0 + r < in.rows && c0 + c < in.cols ? (float)((double)value_of(g + (int64_t)(r0 + r) * in.ld + c0 + c) * scale) : 0.f;
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 512; k += kThreads) {  // 4 x 2 blocks of 64 pieces
        const int row = (k >> 7) * 16 + (k & 15), g8 = k >> 4 & 3, col = (k >> 6 & 1) * 32 + g8 * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = in.tall ? tile[col + j][row] : tile[row][col + j];
        u32x4_t hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t h, l;
            split_f16(v[2 * j], v[2 * j + 1], h, l);
            hi[j] = h, lo[j] = l;
        }
        const int R = (in.tall ? c0 : r0) / 16 + (k >> 7), C = (in.tall ? r0 : c0) / 32 + (k >> 6 & 1);
        if (R >= in.block_rows) continue;
        const int64_t at = matrix * in.x.matrix + ((int64_t)R * in.x.blocks + C) * ORTH_BLOCK + orth_piece(k & 15, g8) * 16;
        *(u32x4_t*)(in.x.part[0] + at) = hi;
        *(u32x4_t*)(in.x.part[1] + at) = lo;
    }
}

// ---- ranges of the operands ----
// The largest power of two from `least` to `most` with which values up to `bound` take half of fp16's range at most.
float scale_for(double bound, float most, float least) {
    const double room = 32752.0 / bound;
    return room >= most ? most : fmaxf((float)exp2(floor(log2(room))), least);
}

// Bounds of a step, from its coefficients and those before it, for any matrix: |G| is at least its largest singular value, so X begins with singular values
// in [0, 1]; on [0, s] those of Q lie in the range of a + b t + c t^2 for t in [0, s^2], and the next X's in that of their products with s.
// An entry of a matrix is at most its largest singular value.  Small singular values (and padded rows) take Q's value at 0, which is a.
// (Steps that lead past all range for some matrix may stay in range for others, and are held for those.)
constexpr int RAISED_MOST = 1 << 10, RAISED_LEAST = -24;
struct Range {
    double most;             // the largest of Q's
    double bound, slope;     // of X before the step; of the slope of a + b t + c t^2
    float x, s, q;           // scales of X before the step, of S and Q
    float from;              // S's over that of X X^T
    int raised;              // X has grown by no more than this power of two
    void coefficients(const float* c, float* abc) const { abc[0] = c[0] * q, abc[1] = c[1] * (q / s), abc[2] = c[2] * (q / (s * s)); }  // of products as they are kept
};
void ranges_of(const float* coefficients, int steps, Range* z) {
    double x = 1, raised = 0;
    for (int k = 0; k < steps; ++k) {
        const double a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2], end = x * x;
        auto q = [&](double t) { return fabs(a + b * t + c * t * t); };
        double most = fmax(q(0), q(end)), next = x * q(end);
        if (c != 0) {
            const double t = -b / (2 * c);  // where Q's has its extreme
            if (t > 0 && t < end) most = fmax(most, q(t));
        }
        // extremes of s q(s^2): a + 3 b t + 5 c t^2 = 0
        const double d = 9 * b * b - 20 * a * c;
        for (int i = 0; i < 2; ++i) {
            const double t = c != 0 ? (d >= 0 ? (-3 * b + (i ? sqrt(d) : -sqrt(d))) / (10 * c) : -1) : b != 0 ? -a / (3 * b) : -1;
            if (t > 0 && t < end) next = fmax(next, sqrt(t) * q(t));
        }
        z[k] = {most, x, fmax(fabs(b), fabs(b + 2 * c * end)), scale_for(x, X_SCALE, X_LEAST), scale_for(2 * end, S_SCALE, S_LEAST), scale_for(most, Q_SCALE, Q_LEAST), 0.f, (int)fmin(ceil(raised), RAISED_MOST)};  // (twice its range for X, so four times for S)
        z[k].from = z[k].s / (z[k].x * z[k].x);
        x = next;
        raised += log2(most);
        if (isnan(raised)) raised = INFINITY;
        if (raised < RAISED_LEAST) raised = RAISED_LEAST;  // (more of a lift is not wanted)
    }
}
// May two steps be taken at a time?  Q' Q is kept times Q_SCALE, and its entries reach |Q'| |Q| (11.9 of the default coefficients, 34 where the first steps raise
// small singular values most).  And S' = Q S Q is off by a share of |Q|^2 |S|, where the S' of a step by itself is off by one of |S'|; Q' takes that times its
// slope, and the next X times s' more: 68 and 98 roundings with the default coefficients, 280 to 403 in the first steps of schedules that raise small ones by 8 and
// keep the largest near 2.  In pairs from the first on (times less, for the range) five of those are 4.8 times as far off as with 32-bit products for 8 x 128 x 256 in
// fp32, by this rule 1.3 (81 and 86 us); 8 x 129 x 9000 2.6 and 0.96 (357 and 379).
bool together(const Range& one, const Range& two) {
    const double q = one.most * one.bound;
    return one.most * two.most * Q_SCALE <= 32752.0 && q * q * two.slope * two.bound <= 128;
}

// ---- plan ----
struct Size {
    int n, m;        // of X, padded
    int tile;        // 256 or 128; 0: all rows and 32 columns at a time (up to 128 rows)
    int parts;       // of the squares
    // Blocks along the rows of X and of S: an odd number, so that the block rows that are loaded together begin in different places of the memory
    // channels' interleaving (a power of two put them all on the same few).
    int xb, sb;
    int64_t x, s;    // bytes of a plane of X and of S
};

constexpr int kUnits = 256;  // compute units

// How the tiles of a launch take their reductions of `steps` blocks: whole ones in full rounds of the `units` workgroups that run at once (two a compute unit,
// one of 256 x 256), those of the last round, or of the only one, in ranges for the places that would have none: four blocks a range at least, and the time
// of 6 saved, about what a second launch costs, and of up to 12 more for the sums' way to memory and back (330 x 826 in fp32, up to 63 ranges that save 8 or more: 187 us,
// whole 222; 16 x 512 x 512 in bf16, 480 ranges that save 11: 288, whole 204; 2 x 600 x 6000 in fp32, 150 that save 16: 380, whole 422).
struct Cut { int whole, splits; };
Cut cut_of(int64_t tiles, int steps, int units) {
    const int rest = (int)(tiles % units), most = steps / 4;
    const int room = rest > 0 ? units / rest : 1, s = room < most ? room : most;
    if (s > 1 && steps - steps / s >= 6 + 12 * rest * s / units) return {(int)(tiles - rest), s};
    return {(int)tiles, 1};
}

// Time of a product's tiles, roughly, in blocks of the reduction of a tile of 256 (0.86 us in one part, 2.2 in two): 8 for a tile's beginning and end, 24 for
// those of a cut one and its sums; a round of small tiles, two a compute unit, 0.6 of one of large ones.
double product_time(int64_t tiles, int64_t steps, int tile) {
    const int units = tile == 256 ? kUnits : 2 * kUnits;
    const Cut c = cut_of(tiles, (int)steps, units);
    return ((double)((c.whole + units - 1) / units) * (steps + 8) + (c.splits > 1 ? (double)steps / c.splits + 24 : 0)) * (tile == 256 ? 1.0 : 0.6);
}
// ... of the products of a step of E matrices: S, its polynomial (any product of squares), the one with X
struct StepTime { double s, square, x; };
StepTime step_time(int E, int n, int m, int tile) {
    const int64_t nt = (n + tile - 1) / tile, mt = (m + tile - 1) / tile, half = nt * (nt + 1) / 2 * E, reduction = nt * tile / 32;
    return {product_time(half, mt * tile / 32, tile), product_time(half, reduction, tile), product_time(nt * mt * E, reduction, tile)};
}
// Large tiles where they take less of that: 128 matrices of 768 x 2048 in bf16 4.3 ms with large ones and 4.8 with small ones, 8 of 1100 x 1300 0.73 and 0.53, one
// of 2048 x 2048 in fp32 0.82 and 0.68.
int tile_of(int E, int n, int m) {
    auto sum = [&](int tile) {
        const StepTime t = step_time(E, n, m, tile);
        return t.s + t.square + t.x;
    };
    return sum(256) < sum(128) ? 256 : 128;
}

Size size_of_matrix(int E, int rows, int cols) {
    Size z;
    const int n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    z.tile = n <= 128 ? 0 : tile_of(E, n, m);
    z.n = z.tile == 0 ? (n <= 32 ? 32 : n <= 64 ? 64 : 128) : (n + z.tile - 1) / z.tile * z.tile;
    z.m = z.tile == 0 ? (m + 63) / 64 * 64 : (m + z.tile - 1) / z.tile * z.tile;
    z.xb = z.m / 32 + 1, z.sb = z.n / 32 + 1;
    z.x = (int64_t)z.n / 16 * z.xb * ORTH_BLOCK;
    z.s = (int64_t)z.n / 16 * z.sb * ORTH_BLOCK;
    const int64_t want = ((int64_t)rows * cols + 16383) / 16384;
    z.parts = (int)(want < 512 ? want : 512);
    if (z.parts > rows) z.parts = rows;
    return z;
}

// X in two parts, twice (one is read while the next is written); S, Q and T in two parts; the partial sums of the squares; the lift
int64_t matrix_bytes(const Size& z) { return 4 * z.x + 6 * z.s + z.n * 8 + 4096 + 16; }
// Workgroups that share the columns of a matrix of up to 128 rows, of which each leaves sums; fewer of the tallest, whose sums are larger
int thin_groups(int count, const Size& z) {
    const int want = z.n == 128 ? (z.m / 32 + 1) / 2 : (z.m / 32 + 3) / 4, room = 2 * kUnits / count > 1 ? 2 * kUnits / count : 1, most = z.n == 128 && room > 128 ? 128 : room;
    return want < most ? want : most;
}
// Sums of the cut reductions of `count` matrices
int64_t part_bytes(int count, const Size& z) {
    if (z.tile == 0) return (int64_t)count * thin_groups(count, z) * z.n * z.n * 4 * 2;
    const int64_t nt = z.n / z.tile, mt = z.m / z.tile, half = nt * (nt + 1) / 2 * count, all = nt * mt * count;
    int64_t most = 0;
    auto product = [&](int64_t tiles, int64_t steps, bool flat) {
        const Cut c = cut_of(tiles, (int)steps, z.tile == 256 && !flat ? kUnits : 2 * kUnits);
        const int64_t bytes = (tiles - c.whole) * c.splits * z.tile * z.tile * (flat ? 2 : 4);
        if (c.splits > 1 && bytes > most) most = bytes;
    };
    product(half, z.m / 32, false);
    product(half, z.n / 32, false);
    product(all, z.n / 32, false);
    if (z.tile == 256) product(2 * all, z.n / 32, true);
    return most;
}
// ... where there are any, at most
constexpr int64_t kPartBytes = (int64_t)kUnits * 256 * 256 * 4;

template <int PA, int PB, bool TB, int CIN, bool ROWS, int PARTS, int OUT> hipError_t product(OrthArgs g, int tile, hipStream_t st) {
    constexpr int PLANES = PA + PB, KS = PLANES == 2 ? 2 : 1, STAGES = PLANES == 2 ? 4 : 2;
    // One-part products with X, whose tiles read X's second part and write both, are cut to 256 x 128 by four wavefronts, two workgroups a unit, of
    // which one multiplies while the other begins or ends a tile: they load half as much again, and 8 x 4096 x 14336 in bf16 takes 30.3 ms
    // instead of 30.9 all the same, 128 x 768 x 2048 4.53 instead of 4.60.  (The products of squares, which write little, are slower so, by 1 %.)
    constexpr bool FLAT = PLANES == 2 && TB;
    const bool flat = FLAT && tile == 256;
    if (flat) g.nt *= 2, g.tiles *= 2;
    const int64_t tiles = (int64_t)g.tiles * g.matrices;
    const Cut c = cut_of(tiles, g.steps, tile == 256 && !flat ? kUnits : 2 * kUnits);
    g.whole = c.whole;
    g.splits = c.splits;
    const int64_t cut = tiles - g.whole;
    auto run = [&](auto kernel, int bytes, int threads) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        kernel<<<g.whole + cut * g.splits, threads, bytes, st>>>(g);
        return hipGetLastError();
    };
    hipError_t e;
    if (tile == 128) e = run(orth_product_kernel<PA, PB, TB, 2, 2, 4, 4, 1, STAGES, CIN, ROWS, PARTS, OUT>, 8 * PLANES * STAGES * ORTH_BLOCK, 256);
    else if constexpr (FLAT) e = run(orth_product_kernel<PA, PB, TB, 2, 2, 8, 4, 1, 3, CIN, ROWS, PARTS, OUT>, 24 * 3 * ORTH_BLOCK, 256);
    else e = run(orth_product_kernel<PA, PB, TB, 2, 4, 8, 4, KS, 2, CIN, ROWS, PARTS, OUT>, 16 * PLANES * KS * 2 * ORTH_BLOCK, 512);
    if (e != hipSuccess || cut == 0) return e;
    if (tile == 128) orth_sums_kernel<8, 8, CIN, ROWS, PARTS, OUT><<<cut * 8, 256, 0, st>>>(g);
    else orth_sums_kernel<16, FLAT ? 8 : 16, CIN, ROWS, PARTS, OUT><<<cut * (FLAT ? 16 : 32), 256, 0, st>>>(g);
    return hipGetLastError();
}

struct Buffers {
    OrthOperand x[2], s, q, t;
    float *part, *own;
    int* lift;
};

OrthOperand operand(char*& at, int64_t plane, int blocks, int matrices) {
    OrthOperand o = {};
    for (int p = 0; p < 2; ++p) {
        o.part[p] = at;
        at += plane * matrices;
    }
    o.matrix = plane;
    o.blocks = blocks;
    return o;
}

// The steps of `count` matrices whose X lies in w.x[0]
template <bool F32> struct Steps {
    const OrthTask& t;
    const Size& z;
    Buffers& w;
    int count;
    void* out;
    hipStream_t st;
    const Range* ranges;  // of each step

    // Steps from k on that are taken at a time where pairs are
    int at_a_time(int k, bool pairs) const { return pairs && k + 2 <= t.steps && together(ranges[k], ranges[k + 1]) ? 2 : 1; }

    OrthArgs square(const OrthOperand& a, const OrthOperand& b, const OrthOperand& c, float alpha) const {  // c = alpha a b, symmetric
        OrthArgs g = {};
        g.matrices = count;
        g.mt = g.nt = z.n / z.tile;
        g.tiles = g.mt * (g.mt + 1) / 2;
        g.a = a, g.b = b, g.c = c;
        g.steps = a.blocks - 1;
        g.alpha = alpha;
        g.part = w.part;
        g.square = z.n;
        g.lift = w.lift, g.sunk_after = RAISED_MOST;  // (taken out of no sums)
        return g;
    }
    // q X of the steps before `next`: into X's other buffer, or to the caller
    void scale(OrthArgs& g, int k, int next, float q) const {
        g.beta = (next < t.steps ? ranges[next].x : t.scale) / ranges[k].x;
        g.alpha = g.beta / q;
        lifted(g, 1, k, next);
    }
    // sums of the X before step k, so many times over, for what is kept before step `next`
    void lifted(OrthArgs& g, int lifts, int k, int next) const {
        g.lift = w.lift, g.lifts = lifts;
        g.sunk = ranges[k].raised, g.sunk_after = next < t.steps ? ranges[next].raised : RAISED_MOST;
    }
    void to_caller(OrthArgs& g) const {
        g.out = out;
        g.out_matrix = t.out_matrix;
        g.out_ld = t.out_ld;
        g.tall = t.rows > t.cols;
        g.rows = g.tall ? t.cols : t.rows;
        g.cols = g.tall ? t.rows : t.cols;
        const int size = F32 ? 4 : 2;
        g.vec = ((uintptr_t)out & (4 * size - 1)) == 0 && t.out_ld % 4 == 0 && (count == 1 || t.out_matrix % 4 == 0);
    }
    // X = q X of the steps from k to next; where q has one part, q of X's first part, what the diagonal's rounding lost of that, and the diagonal's share of X's second
    template <bool TWO> hipError_t apply(const OrthOperand& q, float q_scale, int k, int next) {
        constexpr int PARTS = TWO ? 2 : 1, CIN = TWO ? 0 : 2;
        OrthArgs g = {};
        g.matrices = count;
        g.mt = z.n / z.tile, g.nt = z.m / z.tile;
        g.tiles = g.mt * g.nt;
        g.square = z.n;
        g.a = q, g.b = w.x[0], g.c = w.x[1], g.cin = w.x[0];
        g.own = w.own;
        g.steps = z.n / 32;
        scale(g, k, next, q_scale);
        g.part = w.part;
        hipError_t e;
        if (next < t.steps) {
            e = product<PARTS, PARTS, true, CIN, !TWO, 2, ORTH_BLOCKS>(g, z.tile, st);
        } else {
            to_caller(g);
            e = product<PARTS, PARTS, true, CIN, !TWO, 0, F32 ? ORTH_F32 : ORTH_BF16>(g, z.tile, st);
        }
        const OrthOperand o = w.x[0];
        w.x[0] = w.x[1];
        w.x[1] = o;
        return e;
    }
    // S = X X^T
    hipError_t gram(int k, const Range& r) const {
        constexpr int PARTS = F32 ? 2 : 1;
        OrthArgs g = square(w.x[0], w.x[0], w.s, r.from);
        lifted(g, 2, k, t.steps);
        return product<PARTS, PARTS, false, 0, false, PARTS, ORTH_SQUARE>(g, z.tile, st);
    }
    // to = a I + b S + c S S, and where it has one part its diagonal in 32 bits and what it lost
    hipError_t polynomial(const OrthOperand& to, int k, const Range& r) const {
        constexpr int PARTS = F32 ? 2 : 1;
        float abc[3];
        r.coefficients(t.coefficients + 3 * k, abc);
        OrthArgs g = square(w.s, w.s, to, abc[2]);
        g.cin = w.s;
        g.beta = abc[1];
        g.diagonal = abc[0];
        g.unscale = 1.f / r.q;
        g.own = F32 ? nullptr : w.own;
        return product<PARTS, PARTS, false, PARTS, false, PARTS, ORTH_SQUARE>(g, z.tile, st);
    }
    // to = a b times alpha, of matrices that commute but for rounding
    hipError_t times(const OrthOperand& a, const OrthOperand& b, const OrthOperand& to, float alpha) const {
        return product<2, 2, false, 0, false, 2, ORTH_SQUARE>(square(a, b, to, alpha), z.tile, st);
    }
    hipError_t one_step(int k) {
        const Range& r = ranges[k];
        hipError_t e = gram(k, r);
        if (e == hipSuccess) e = polynomial(w.q, k, r);
        if (e == hipSuccess) e = apply<F32>(w.q, r.q, k, k + 1);
        return e;
    }
    // S of both steps by the scale that holds both
    void pair(int k, Range& one, Range& two) const {
        one = ranges[k], two = ranges[k + 1];
        one.s = two.s = fminf(one.s, two.s);
        one.from = one.s / (one.x * one.x);
    }
    hipError_t two_steps(int k) {
        Range one, two;
        pair(k, one, two);
        hipError_t e = gram(k, one);
        if (e == hipSuccess) e = polynomial(w.q, k, one);
        // (Q X) (Q X)^T = Q S Q in this order: Q's own rounding does not commute with S, and S Q Q is further from it (steps 4 and 5 of those that raise by 8, 768 x
        // 2048: 1.2e-5 off, so 5e-6)
        if (e == hipSuccess) e = times(w.q, w.s, w.t, 1.f / one.q);
        if (e == hipSuccess) e = times(w.t, w.q, w.s, 1.f / one.q);
        if (e == hipSuccess) e = polynomial(w.t, k + 1, two);
        if (e == hipSuccess) e = times(w.t, w.q, w.s, Q_SCALE / (one.q * two.q));
        if (e == hipSuccess) e = apply<true>(w.s, Q_SCALE, k, k + 2);
        return e;
    }
    // Two steps' Q in one launch
    template <int NF> hipError_t link(float* sums, const OrthArgs& of, int k) {
        OrthArgs g = {};
        g.part = sums;
        g.c = w.q;
        lifted(g, 2, k, t.steps);
        Range one, two;
        pair(k, one, two);
        OrthPair p = {};
        p.from = one.from, p.through = 1.f / one.q, p.joint = Q_SCALE / (one.q * two.q);
        one.coefficients(t.coefficients + 3 * k, p.abc[0]);
        two.coefficients(t.coefficients + 3 * k + 3, p.abc[1]);
        constexpr int bytes = 4 * NF * (NF / 2) * ORTH_BLOCK;
        auto kernel = orth_chain_kernel<NF>;
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        kernel<<<count, NF * 64, bytes, st>>>(g, of.apart, of.ranges, p);
        return hipGetLastError();
    }
    // Matrices of up to 128 rows (16 NF padded)
    template <int NF, int MODE, int OUT, bool OWN> static auto step_kernel() {
        if constexpr (NF == 8) return orth_rows_kernel<MODE, OUT, OWN>;
        else return orth_thin_kernel<NF, MODE, OUT, OWN>;
    }
    template <int NF> hipError_t thin() {
        const int groups = thin_groups(count, z);
        auto launch = [&](auto kernel, const OrthArgs& g, bool own) {
            const int bytes = ((NF == 8 ? 6 * NF : 4 * (NF * NF > 2 * NF ? NF * NF : 2 * NF)) + (own ? NF * NF : 0)) * ORTH_BLOCK;
            const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
            if (e != hipSuccess) return e;
            kernel<<<dim3(groups, count), 256, bytes, st>>>(g);
            return hipGetLastError();
        };
        OrthArgs g = {};
        g.matrices = count;
        g.a = w.q, g.b = w.x[0];
        g.steps = z.m / 32;
        float *sums = w.part, *next = w.part + part_bytes(count, z) / 8;  // (read and written by one launch)
        g.part = sums;
        hipError_t e = launch(step_kernel<NF, 0, ORTH_BLOCKS, false>(), g, false);
        // Small matrices have few values to average over, and 32-bit products lose little on them: fp32 results keep up with those up to 64 rows where steps are
        // taken one by one (2 x 24 x 24: 1.1 to 1.2 times their error, 1.7 to 1.9 in pairs).  Otherwise pairs, whose products take a launch of their own, where X is long
        // or Q larger (8 x 16 x 14336 in bf16: 65 us in pairs, 83 one by one; 8 x 128 x 256: 85 and 95).
        const bool pairs = NF == 8 || (!F32 && groups > 8);
        for (int k = 0; k < t.steps && e == hipSuccess;) {
            const int n = at_a_time(k, pairs);
            // many ranges are added in a launch of their own, from more of the larger sums on (8 x 100 x 500, 8 of them: 100 us with it, 121 without; 64 x 64 x 300,
            // 3: 84 and 77; 8 x 64 x 2000, 16: 54 and 60)
            g.apart = g.ranges = groups;
            if (groups > (NF == 8 ? 4 : 8)) {
                orth_fold_kernel<<<dim3(NF * NF / 4, count), 256, 0, st>>>(sums, groups, NF * NF);
                e = hipGetLastError();
                g.ranges = 1;
            }
            if (n == 2 && e == hipSuccess) e = link<NF>(sums, g, k);
            if (e != hipSuccess) break;
            g.sums = sums, g.part = next;
            ranges[k].coefficients(t.coefficients + 3 * k, g.abc);
            g.from = ranges[k].from;
            g.b = w.x[0], g.c = w.x[1];
            scale(g, k, k + n, n == 2 ? Q_SCALE : ranges[k].q);
            k += n;
            constexpr int OUT = F32 ? ORTH_F32 : ORTH_BF16;
            if (k < t.steps) {
                e = n == 2 ? launch(step_kernel<NF, 1, ORTH_BLOCKS, false>(), g, false) : launch(step_kernel<NF, 1, ORTH_BLOCKS, true>(), g, true);
            } else {
                to_caller(g);
                e = n == 2 ? launch(step_kernel<NF, 2, OUT, false>(), g, false) : launch(step_kernel<NF, 2, OUT, true>(), g, true);
            }
            const OrthOperand o = w.x[0];
            w.x[0] = w.x[1];
            w.x[1] = o;
            float* p = sums;
            sums = next;
            next = p;
        }
        return e;
    }
    hipError_t run() {
        if (z.tile == 0) return z.n == 32 ? thin<2>() : z.n == 64 ? thin<4>() : thin<8>();
        // Two steps at a time take S = X X^T and the product with X once, for three more products of squares: less where X is wide (32 x 7168 x 2048 29.9 ms, one by
        // one 38.7; 330 x 826, with its reductions of squares whole, 266 and 223 us).  (With operands in one part the squares would need two and cost more than that gains.)
        const StepTime time = step_time(count, z.n, z.m, z.tile);
        const bool pairs = F32 && time.s + time.x > 3 * time.square;
        hipError_t e = hipSuccess;
        for (int k = 0; k < t.steps && e == hipSuccess;) {
            const int n = at_a_time(k, pairs);
            if constexpr (F32) e = n == 2 ? two_steps(k) : one_step(k);
            else e = one_step(k);
            k += n;
        }
        return e;
    }
};

}  // namespace

// A few matrices at a time where the whole stack would take more than this
constexpr int64_t ORTH_WORKSPACE = (int64_t)8 << 30;

int at_once(int E, const Size& z) {
    const int64_t n = (ORTH_WORKSPACE - kPartBytes) / matrix_bytes(z);
    return n < 1 ? 1 : n < E ? (int)n : E;
}

size_t orth_workspace(int E, int rows, int cols) {
    const Size z = size_of_matrix(E, rows, cols);
    const int turn = at_once(E, z);
    return (size_t)(turn * matrix_bytes(z) + (turn < E ? kPartBytes : part_bytes(E, z)));
}

hipError_t launch_orth(const OrthTask& t, void* workspace, hipStream_t st) {
    const Size z = size_of_matrix(t.E, t.rows, t.cols);
    const int turn = at_once(t.E, z);
    const int64_t part = turn < t.E ? kPartBytes : part_bytes(t.E, z);
    const bool tall = t.rows > t.cols;
    const int size_in = t.in_f32 ? 4 : 2, size_out = t.out_f32 ? 4 : 2;
    Range ranges[ORTH_MAX_STEPS];
    ranges_of(t.coefficients, t.steps, ranges);
    for (int e0 = 0; e0 < t.E; e0 += turn) {
        const int count = t.E - e0 < turn ? t.E - e0 : turn;
        char* at = (char*)workspace;
        Buffers w;
        w.part = (float*)at;
        at += part;
        for (OrthOperand& x : w.x) x = operand(at, z.x, z.xb, count);
        for (OrthOperand* o : {&w.s, &w.q, &w.t}) *o = operand(at, z.s, z.sb, count);
        OrthIn in = {};
        in.g = (const char*)t.g + e0 * t.g_matrix * size_in;
        in.matrix = t.g_matrix;
        in.ld = t.g_ld;
        in.rows = t.rows;
        in.cols = t.cols;
        w.own = (float*)at;
        in.partials = (double*)(at + (int64_t)z.n * 8 * count);
        in.lift = w.lift = (int*)(at + (int64_t)(z.n * 8 + 4096) * count);
        in.parts = z.parts;
        in.eps = t.eps;
        in.tall = tall;
        in.vec = ((uintptr_t)in.g & 15) == 0 && t.g_ld * size_in % 16 == 0 && (count == 1 || t.g_matrix * size_in % 16 == 0);
        in.x = w.x[0];
        in.block_rows = z.n / 16;
        const dim3 blocks(((tall ? z.n : z.m) + 63) / 64, ((tall ? z.m : z.n) + 63) / 64, count);
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
        e = t.out_f32 ? Steps<true>{t, z, w, count, out, st, ranges}.run() : Steps<false>{t, z, w, count, out, st, ranges}.run();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
