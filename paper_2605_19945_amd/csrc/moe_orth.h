// Tile engine of the orthogonalising products (moe_orth.hip): one workgroup computes a tile C[i][j] = sum_k A[i][k] B[j][k] of one matrix.
//
// Operands are matrices of this unit's own making, kept as the matrix instructions read them: 16 rows by 32 columns are a block of 1 KiB, in
// which 8 neighbouring columns of a row are a piece of 16 bytes; blocks follow each other along the columns.  A load into LDS is one block,
// whole lines of memory.  Fragments whose reduction runs along the columns are 16-byte LDS reads, those whose reduction runs along the
// rows come from the transposing 8-byte read, so a matrix is kept once whichever way it is multiplied.  A block's pieces are placed (orth_piece)
// so that both reads fall on all banks.  Rows and columns are padded with zeros to whole tiles, so there are no edges.
//
// Values are held as fp16 times a power of two, as one part (11 bits) or as two whose sum has 22: v = hi + lo, hi = fp16(v), lo = fp16(v - hi).
// A product of such parts takes hi hi, hi lo and lo hi (what there is of them; lo lo lies below the 32-bit sums' rounding).
#pragma once
#include "moe_ops.h"

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char orth_lds_char;

constexpr int ORTH_BLOCK = 1024;  // bytes of a block of 16 rows by 32 values

// A stack of matrices in blocks, one plane a part
struct OrthOperand {
    char* part[2];
    int64_t matrix;  // bytes from one matrix to the next
    int blocks;      // along the columns
};

struct OrthArgs {
    OrthOperand a, b;
    OrthOperand cin;       // beta times this is added, or times the row's of
    float* own;            // of a symmetric result in one part: [matrices][its rows][what its diagonal's rounding lost, its diagonal]
    OrthOperand c;         // the result
    float alpha, beta;
    float diagonal;        // added to the diagonal of a symmetric result
    float unscale;         // ... times this
    const int* lift;       // of each matrix: X is kept times 2 to this power, less `sunk` (at least 0), on top of its scale; the result less `sunk_after`
    int lifts, sunk, sunk_after;  // lifts: how many of them the sums have
    int square;            // rows of a symmetric operand
    int steps;             // blocks of the reduction
    int whole;             // of all matrices' tiles the first `whole` take their reduction whole; the others' is cut into `splits` ranges, whose
    int splits;            // sums go to `part`: [those tiles][splits][fragments of a tile][64 lanes][4]
    float* part;
    int mt, nt;            // tiles of a matrix (symmetric: mt == nt, those on and above the diagonal)
    int tiles, matrices;   // tiles of a matrix that are computed
    // of matrices of up to 128 rows: S in `ranges` sums, `apart` of them a matrix, of which the coefficients give Q
    const float* sums;
    int ranges, apart;
    float from, abc[3];    // S = from times the sums; Q = a I + b S + c S S of S and Q as they are kept
    // the last product: results in the caller's rows
    void* out;
    int64_t out_matrix, out_ld;  // values from one matrix, one row to the next
    int rows, cols;              // of C that exist
    int tall;                    // C is the transpose of what the caller has
    int vec;                     // groups of 4 values are aligned
};

// Two steps at a time, of matrices of up to 128 rows: as from and abc above; S Q's and Q S Q's products times `through`, Q' Q's times `joint`
struct OrthPair {
    float from, abc[2][3], through, joint;
};

enum { ORTH_SQUARE = 0, ORTH_BLOCKS = 1, ORTH_BF16 = 2, ORTH_F32 = 3 };

// Place of a piece in its block: 8 columns from 8 * g on of a row.  A 16-byte read serves lanes 0-3, 12-15 and 20-27 together, the rows 0-3 and 12-15
// of one g and 4-11 of the next; a transposing read the rows 0-3 and 8-11 (or 4-7 and 12-15) of two neighbouring g.  Rows change places by 12 in
// every other g, so that both find 16 pieces of different banks.
static __device__ __host__ inline int orth_piece(int row, int g) { return 16 * g + (row ^ (g & 1) * 12); }

static __device__ inline uint32_t orth_lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const orth_lds_char*)p; }

static __device__ inline u32x4_t orth_desc(const char* base, uint32_t bytes) {
    const uint64_t p = (uint64_t)base;
    u32x4_t d;
    d[0] = __builtin_amdgcn_readfirstlane((uint32_t)p);
    d[1] = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32) & 0xffffu);
    d[2] = __builtin_amdgcn_readfirstlane(bytes);
    d[3] = 0x00027000u;
    return d;
}

// 16 bytes a lane from memory to LDS at `to` + 16 * lane, in asm so that the compiler does not wait for it at the next LDS read; it has no
// output registers.
static __device__ inline void orth_load(uint32_t to, uint32_t offset, const u32x4_t& desc, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(offset), "s"(desc), "s"(at) : "memory");
}
template <int N> static __device__ inline void orth_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
static __device__ inline void orth_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

static __device__ inline uint32_t pack_f16(float lo, float hi) {
    typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
    const f16x2_t v = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
static __device__ inline float f16_lo(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)w); }
static __device__ inline float f16_hi(uint32_t w) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16)); }
// Two values' first parts and second ones.  The first are hidden from the compiler before the second are formed: it would make those from another rounding of
// the values, by an instruction that multiplies, adds and rounds once, which differs in one of some thousand values, by a whole step of the first part.
static __device__ inline void split_f16(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack_f16(x, y);
    asm("" : "+v"(hi));
    lo = pack_f16(x - f16_lo(hi), y - f16_hi(hi));
}

template <int I> struct OrthInt { static constexpr int value = I; };
template <int N, int I = 0, typename F> static __device__ inline void orth_repeat(F&& f) {  // f(0) .. f(N - 1), each a constant
    if constexpr (I < N) {
        f(OrthInt<I>{});
        orth_repeat<N, I + 1>(f);
    }
}

// From the lane 1 (STEP 1) or 2 further on or back among 4
template <int STEP> static __device__ inline uint32_t lane_xor(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, STEP == 1 ? 0xb1 : 0x4e, 0xf, 0xf, false);
}

// 4 lanes have 4 fp16 values each (of row lane % 4, columns 0..3): afterwards each has column lane % 4 of the rows 0..3
static __device__ inline void turn_f16(uint32_t& a, uint32_t& b, int lane) {
    const int t = lane & 3;
    // pairs of lanes: a = (c0, c1) and b = (c2, c3) of one row -> one column of two rows
    const uint32_t xa = lane_xor<1>(a), xb = lane_xor<1>(b);
    const uint32_t a1 = t & 1 ? (xa >> 16) | (a & 0xffff0000u) : (a & 0xffffu) | (xa << 16);
    const uint32_t b1 = t & 1 ? (xb >> 16) | (b & 0xffff0000u) : (b & 0xffffu) | (xb << 16);
    // pairs of pairs: a1 has rows 2p, 2p + 1 of column t % 2, b1 of column 2 + t % 2
    const uint32_t ya = lane_xor<2>(a1), yb = lane_xor<2>(b1);
    a = t & 2 ? yb : a1;
    b = t & 2 ? b1 : ya;
}
static __device__ inline void turn_f32(f32x4_t& v, int lane) {
    const int t = lane & 3;
    // even lanes keep column 0 (2), odd ones 1 (3): lane t has (own, neighbour's) of that column
    const float o0 = __uint_as_float(lane_xor<1>(__float_as_uint(v[0]))), o1 = __uint_as_float(lane_xor<1>(__float_as_uint(v[1])));
    const float o2 = __uint_as_float(lane_xor<1>(__float_as_uint(v[2]))), o3 = __uint_as_float(lane_xor<1>(__float_as_uint(v[3])));
    const float a0 = t & 1 ? o1 : v[0], a1 = t & 1 ? v[1] : o0;  // rows 2p, 2p + 1 of column t % 2
    const float b0 = t & 1 ? o3 : v[2], b1 = t & 1 ? v[3] : o2;  // of column 2 + t % 2
    const float ya0 = __uint_as_float(lane_xor<2>(__float_as_uint(a0))), ya1 = __uint_as_float(lane_xor<2>(__float_as_uint(a1)));
    const float yb0 = __uint_as_float(lane_xor<2>(__float_as_uint(b0))), yb1 = __uint_as_float(lane_xor<2>(__float_as_uint(b1)));
    v = t & 2 ? f32x4_t{yb0, yb1, b0, b1} : f32x4_t{a0, a1, ya0, ya1};
}
