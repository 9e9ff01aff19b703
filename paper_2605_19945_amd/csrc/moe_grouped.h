// Tile engine of the matrix products grouped by expert (moe_grouped_gemm, moe_grouped_gemm_wgrad,
// moe_mxfp4_grouped_gemm): one workgroup computes a BM x BN tile C[m][n] = sum_k A[m][k] B[n][k] of one expert.
//
// An operand lies in memory either with the reduction index contiguous (LAY_K: a row of the tile is one m or n) or
// with m or n contiguous (LAY_MN: a row of the tile is one k).  Forward products read rows in LAY_K and row-major
// weights [K, N] in LAY_MN, the gradient of the rows reads both in LAY_K, the gradient of the weights both in LAY_MN.
// Both kinds are staged as they lie: a K step is 128 bytes of every LAY_K row (64 bf16 or 256 4-bit values) or 64 LAY_MN rows,
// and goes from memory into LDS directly.  A LAY_K fragment is a 16-byte LDS read; a LAY_MN fragment is turned by the
// transposing 8-byte LDS read, so neither layout needs a transposed copy in memory.
//
// Edges cost no code in the loop: loads go through a buffer descriptor that ends at the tile's last valid row, and lanes
// whose column is none get an offset behind it; both read zeros.  So a last K step of any length is zeros times zeros.
#pragma once
#include "moe_internal.h"

enum { FMT_BF16 = 0, FMT_MX4 = 1 };
enum { LAY_K = 0, LAY_MN = 1 };
enum { OUT_BF16 = 0, OUT_F32 = 1, OUT_F32_ADD = 2 };

struct GroupedArgs {
    const char* a;           // rows operand, or x of the weight gradient
    const char* b;           // weights, or dy of the weight gradient
    const uint8_t* sa;       // block scales of a and b (FMT_MX4)
    const uint8_t* sb;
    void* c;
    const int32_t* offsets;  // [E + 1]
    int64_t lda, ldb, ldc;   // bytes between rows of a and b, values between rows of c
    int64_t b_expert;        // bytes between the experts' weights
    int E, rows_cap;
    int M, N;                // M: width of x in the weight gradient (otherwise the experts' rows)
    int kbytes;              // bytes of a LAY_K row; values of the reduction where no operand is LAY_K (0: an expert's rows)
    int scale_ld;            // bytes between rows of scales
    int splits;              // ranges the reduction is cut into (1: none)
    float* part;             // their partial sums, laid out like c without gaps (rows N values apart), one slab after the other
    int64_t slab;            // values of a slab
};

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;  // an offset behind the end of every descriptor (those are below 2 GB)

static __device__ inline uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const lds_char*)p; }

static __device__ inline u32x4_t make_desc(const char* base, int bytes) {
    const uint64_t p = (uint64_t)base;
    u32x4_t d;
    d[0] = __builtin_amdgcn_readfirstlane((uint32_t)p);
    d[1] = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32) & 0xffffu);
    d[2] = __builtin_amdgcn_readfirstlane(max(bytes, 0));
    d[3] = 0x00027000u;
    return d;
}

// 16 bytes a lane from memory to LDS at `to` + 16 * lane.  Inline asm, so that the compiler does not wait for it at the
// next LDS read; it has no output registers.
// NT: with the non-temporal hint, for weights that one workgroup reads once.
template <bool NT = false> static __device__ inline void load_to_lds(uint32_t to, uint32_t offset, const u32x4_t& desc) {
    if (NT) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(offset), "s"(desc) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(desc) : "memory");
}
template <int N> static __device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
static __device__ inline void block_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Rows [lo, lo + n) of expert e, cut to [0, cap): offsets that do not ascend or pass the bound never lead out of it.
static __device__ inline void expert_rows(const int32_t* offsets, int e, int cap, int* lo, int* n) {
    const int a = min(max(offsets[e], 0), cap), b = min(max(offsets[e + 1], 0), cap);
    *lo = a;
    *n = max(b - a, 0);
}

struct GroupedTile {
    int e, lo, n;  // expert, its first row, its rows
    int m0, n0;    // first row (column of x in the weight gradient) and first column of the tile
    int split;     // range of the reduction
    int pieces;    // ranges that its reduction is cut into
    int rows;      // rows (columns of x) of the tile that exist
};

// Inside one expert's mt x nt tiles: bands of up to BAND row tiles, row tiles fastest, so that the 32 compute units of an XCD work
// on neighbouring tiles and share their panels in its L2: about 8 x 4 of them, in the gradient of the weights 5 x 6 (128 experts, 2048 x
// 1536 from 65528 rows 723 -> 662 us, 32 experts, 2048 x 7168 from 5003 rows 415 -> 319; row products are the same within 1 % at 4, 6, 8, 12).
template <int BAND> static __device__ inline void place_in_band(int t, int mt, int nt, int* m, int* n) {
    const int band = t / (BAND * nt), r = t - band * BAND * nt;
    const int h = min(BAND, mt - BAND * band);
    *n = r / h;
    *m = BAND * band + r - *n * h;
}

// The list of the row tiles (BM rows) of all experts times nt column tiles times the ranges of the reduction, kept by every wave
// in its registers, 4 experts a lane; each XCD (workgroup number % 8) takes one stretch [begin, end) of it.
template <int BM> struct RowTiles {
    int lo[4], n[4], cnt[4], before, upto;  // row tiles before the lane's experts, and with them
    int nt, begin, end;

    __device__ inline void init(const GroupedArgs& g, int nt_, int splits) {
        const int lane = threadIdx.x & 63;
        nt = nt_;
        before = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 4 * lane + j;
            lo[j] = n[j] = 0;
            if (e < g.E) expert_rows(g.offsets, e, g.rows_cap, &lo[j], &n[j]);
            cnt[j] = (n[j] + BM - 1) / BM;
            before -= cnt[j];
        }
        upto = -before;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        before += upto;
        int64_t total = (int64_t)__builtin_amdgcn_readlane(upto, 63) * nt * splits;
        if (total > 0x7fffffff) total = 0;  // (overlapping experts only: the offsets are none)
        const int xcd = blockIdx.x & 7;
        begin = (int)(total * xcd / 8);
        end = (int)(total * (xcd + 1) / 8);
    }
    __device__ inline GroupedTile find(int t, int bn, int splits) const {
        GroupedTile out = {};
        out.split = t % splits;
        t = t / splits;
        const int tm = __builtin_amdgcn_readfirstlane(t / nt);  // an expert's tiles are its row tiles times nt
        const int src = __builtin_ctzll(__ballot(upto > tm));
        int b = __builtin_amdgcn_readlane(before, src), mt = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = __builtin_amdgcn_readlane(cnt[j], src);
            if (mt == 0) {
                if (tm < b + c) {
                    mt = c;
                    out.e = 4 * src + j;
                    out.lo = __builtin_amdgcn_readlane(lo[j], src);
                    out.n = __builtin_amdgcn_readlane(n[j], src);
                } else {
                    b += c;
                }
            }
        }
        int m, c;
        place_in_band<8>(t - b * nt, mt, nt, &m, &c);
        out.m0 = __builtin_amdgcn_readfirstlane(m) * BM;
        out.n0 = __builtin_amdgcn_readfirstlane(c) * bn;
        return out;
    }
};

// The list of all tiles, expert by expert, follows from the offsets alone; each XCD (workgroup number % 8) takes one stretch of
// it, and its workgroups go through that side by side.  Every workgroup builds what it needs of the list in LDS.
struct TileList {
    int lo[256], n[256];  // first row and rows of every expert
    int first[257];       // row tiles before the expert (products over ragged rows)
    int begin, end;       // this XCD's stretch
    int height;           // rows of a tile (products over ragged rows)
    int pieces, whole, rest;  // tiles [whole, whole + rest) of the stretch are cut into `pieces` ranges, one a workgroup
};

// Cost of a tile of a weight gradient beside its K steps, in K steps: its stores (32 experts, 2048 x 7168 from 5003 rows 300 / 323 / 392
// us with 4 / 6 / 12, 128 experts, 2048 x 1536 from 65528 rows 671 / 664 with 4 / 6).
constexpr int TILE_COST = 5;
// Time of a K step of a tile over ragged rows: a share for every quarter of its height, and one beside (the columns, the barriers and
// most of the loads' latency: the gradient of 65536 rows of 128 experts 429 us with 2 and 22 or 4 and 14, 441 with 5 and 7; 10432 to 3272,
// one expert, 7748 rows, whose last round can be cut at three quarters of the height, 465 with 2 and 22, 508 with 4 and 14).
constexpr int QUARTER_COST = 2, STEP_COST = 22;

// TAIL: the last round of tiles of 256 rows seldom fills the card.  Where it takes half of an XCD's workgroups or fewer, the
// reductions of its tiles are cut into ranges for the others too, each leaves its sums in a slot of the workspace, and a second kernel
// adds them in their order.  PIECE_COST: of a range's way to memory and back, on an XCD.
constexpr int SIDE = 32;  // workgroups of an XCD
constexpr int PIECE_COST = 17;
constexpr int64_t PIECE = 256 * 256;  // values of a slot

// By one wave.  An entry is a tile and a range of its reduction.  WEIGHTS: every expert has `per` entries, which cost what it
// has rows, and the stretches are of equal cost; otherwise a tile costs the same everywhere.
template <bool WEIGHTS, int BM, bool TAIL> static __device__ inline void make_list(const GroupedArgs& g, int per, TileList* l) {
    const int lane = threadIdx.x & 63, xcd = blockIdx.x & 7;
    int rows[4], c[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = 4 * lane + j;
        int lo = 0;
        rows[j] = 0;
        if (e < g.E) expert_rows(g.offsets, e, g.rows_cap, &lo, &rows[j]);
        l->lo[e] = lo;
        l->n[e] = rows[j];
    }
    int height = BM, pieces = 1;
    if (!WEIGHTS) {
        // Quarters of BM in the height that leaves the least to the busiest workgroup.  A step of a tile takes QUARTER_COST for every
        // quarter and STEP_COST beside.
        int64_t best = INT64_MAX;
#pragma unroll
        for (int quarters = 4; quarters > 0; --quarters) {
            const int h = BM / 4 * quarters;
            int tiles = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) tiles += (rows[j] + h - 1) / h;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) tiles += __shfl_xor(tiles, d);
            const int step = STEP_COST + QUARTER_COST * quarters;
            if constexpr (TAIL) {
                const uint32_t steps = (g.kbytes + 127) / 128, most = (uint32_t)min(((int64_t)tiles * per + 7) / 8, (int64_t)0x7fffffff);
                const uint32_t full = most / SIDE, rest = most % SIDE;
                int64_t cost = (int64_t)(full + (rest > 0)) * steps * step;
                int cut = 1;
                if (rest > 0 && rest <= SIDE / 2) {
                    for (uint32_t s = min(SIDE / rest, steps / 4); s > 1; s = s * 3 / 4) {
                        const int64_t other = ((int64_t)full * steps + (steps + s - 1) / s) * step + PIECE_COST * (int)(rest * s);
                        if (other < cost) {
                            cost = other;
                            cut = (int)s;
                        }
                    }
                }
                if (cost < best) {
                    best = cost;
                    height = h;
                    pieces = cut;
                }
            } else {
                const int64_t cost = ((int64_t)tiles * per + gridDim.x - 1) / gridDim.x * step;
                if (cost < best) {
                    best = cost;
                    height = h;
                }
            }
        }
        height = __builtin_amdgcn_readfirstlane(height);
        if (lane == 0) l->height = height;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c[j] = WEIGHTS ? (4 * lane + j < g.E ? (rows[j] + 63) / 64 + TILE_COST : 0) : (rows[j] + height - 1) / height;
        sum += c[j];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    const int all = __builtin_amdgcn_readlane(incl, 63);
    int before = incl - sum;
    int64_t total = (int64_t)all * per;
    if (!WEIGHTS && total > 0x7fffffff) total = 0;  // (overlapping experts only: the offsets are none)
    // the first tile at or behind position `at` of the total cost (of expert e: at = per * before + tile * c)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t at = total * (xcd + k) / 8;
        if (!WEIGHTS) {
            if (lane == 0) (k ? l->end : l->begin) = (int)at;
        } else if (xcd + k == 8) {
            if (lane == 0) l->end = g.E * per;
        } else {
            int b = before;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t from = (int64_t)b * per, to = from + (int64_t)c[j] * per;
                if (c[j] > 0 && at >= from && at < to) (k ? l->end : l->begin) = (4 * lane + j) * per + (int)((at - from + c[j] - 1) / c[j]);
                b += c[j];
            }
        }
    }
    if (TAIL && lane == 0) {  // (an XCD's rest is that of the longest stretch or one less)
        const int begin = (int)(total * xcd / 8), n = (int)(total * (xcd + 1) / 8) - begin, rest = n % SIDE;
        l->pieces = pieces;
        l->rest = rest;
        l->whole = begin + n - rest;
        if (pieces > 1) l->end = begin + n - rest + rest * pieces;
    }
    if (!WEIGHTS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            l->first[4 * lane + j] = before;
            before += c[j];
        }
        if (lane == 63) l->first[256] = before;
    }
}

template <bool WEIGHTS, int BM, int BN, bool TAIL>
static __device__ inline GroupedTile find_tile(const GroupedArgs& g, const TileList& l, int splits, int height, int mt, int nt, int t) {
    GroupedTile out;
    int e, m, n, r;
    out.split = t % splits;
    out.pieces = splits;
    t = __builtin_amdgcn_readfirstlane(t / splits);
    if (TAIL) {
        const int j = t - l.whole, pieces = l.pieces;
        if (pieces > 1 && j >= 0) {  // a range of a tile
            out.pieces = __builtin_amdgcn_readfirstlane(pieces);
            out.split = __builtin_amdgcn_readfirstlane((uint32_t)j / l.rest);
            t = __builtin_amdgcn_readfirstlane(l.whole + (uint32_t)j % l.rest);
        }
    }
    if (WEIGHTS) {
        e = __builtin_amdgcn_readfirstlane(t / (mt * nt));
        r = t - e * mt * nt;
    } else {
        const int tm = __builtin_amdgcn_readfirstlane(t / nt);  // an expert's tiles are its row tiles times nt
        const uint64_t past = __ballot(l.first[4 * (threadIdx.x & 63) + 4] > tm);
        e = 4 * __builtin_ctzll(past);
        e += (l.first[e + 1] <= tm) + (l.first[e + 2] <= tm) + (l.first[e + 3] <= tm);
        e = __builtin_amdgcn_readfirstlane(e);
        r = t - l.first[e] * nt;
        mt = l.first[e + 1] - l.first[e];
    }
    r = __builtin_amdgcn_readfirstlane(r);
    mt = __builtin_amdgcn_readfirstlane(mt);
    place_in_band<WEIGHTS ? 5 : 8>(r, mt, nt, &m, &n);
    out.e = e;
    out.lo = __builtin_amdgcn_readfirstlane(l.lo[e]);
    out.n = __builtin_amdgcn_readfirstlane(l.n[e]);
    m = __builtin_amdgcn_readfirstlane(m);
    if (WEIGHTS) {
        out.m0 = m * height;
        out.rows = min(g.M - out.m0, height);
    } else {  // the expert's rows are cut evenly, in quarters of the tallest tile: neighbours that share a panel stay side by side
        const int q = (out.n + BM / 4 - 1) / (BM / 4), each = q / mt, over = q - each * mt;
        const int from = __builtin_amdgcn_readfirstlane(m * each + min(m, over)), to = __builtin_amdgcn_readfirstlane((m + 1) * each + min(m + 1, over));
        out.m0 = from * (BM / 4);
        out.rows = min(out.n, to * (BM / 4)) - out.m0;
    }
    out.n0 = __builtin_amdgcn_readfirstlane(n) * BN;
    return out;
}

// 16-byte chunk c of a row lies at chunk c ^ swizzle(row) of its LDS row, so that the lanes that read together fall on
// different banks.  LAY_MN: rows 0-3 and 8-11, two neighbouring chunks.  LAY_K: a 16-byte read serves lanes 0-3, 12-15 and 20-27 together,
// so rows 0-3 and 12-15 of one chunk (swizzles 0 to 3) and rows 4-11 of a second one (4 to 7): whichever two chunks of an even distance
// below 4 or neighbouring ones those are, the two sets stay apart (no conflicts counted for either format).
// Rows of 64 bytes lie four to a turn of the banks, so the four rows that share a place in it need a chunk each.
template <int SPAN> static __device__ inline int swizzle_k(int row) {
    if (SPAN == 64) {
        const int t = row >> 2;
        return (t << 1 & 2) ^ (t & 2) ^ (t >> 1 & 1);  // 0, 2, 3, 1 for t = 0 .. 3
    }
    const int t = row >> 1;
    return (t & 1) | (t >> 1 & 2) | ((t ^ t << 1) & 4);
}

// Rows of 64 columns lie two to a turn of the banks.
template <int B> static __device__ inline int swizzle_mn(int row) {
    return B == 64 ? (row & 2) | (row >> 1 & 4) : 2 * ((row & 3) + (row >> 1 & 4));
}

// One operand's share of a wave: NL loads of 1 KiB a stage.  A stage is SPAN bytes of LAY_K rows or SPAN / 2 LAY_MN rows.
template <int LAY, int B, int NL, int SPAN = 128> struct Loader {
    static constexpr int ROW = LAY == LAY_K ? SPAN : 2 * B;  // bytes of a row in LDS
    const char* base;
    int64_t step;        // bytes to the next K step
    uint32_t ld;         // bytes between rows
    int width;           // bytes of the last row that belong to the operand
    int rows;            // LAY_K: valid rows of the tile; LAY_MN: rows (k) left from this step on
    uint32_t offset[NL];

    // `first`: the address of the tile's first value; `valid`: rows (LAY_K) or columns (LAY_MN) of the tile that exist;
    // `k`: bytes (LAY_K) or rows (LAY_MN) of the reduction
    __device__ inline void init(const char* first, int64_t ld_, int valid, int k, int wave) {
        const int lane = threadIdx.x & 63;
        base = first;
        ld = (uint32_t)ld_;
        if (LAY == LAY_K) {
            step = SPAN;
            rows = min(valid, B);
            width = k;
        } else {
            step = SPAN / 2 * ld_;
            rows = k;
            width = 2 * max(min(valid, B), 0);  // (none in the lower half of a low tile)
        }
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int p = (wave * NL + j) * 1024 + lane * 16;
            const int row = p / ROW, chunk = (p % ROW) / 16;
            const int c = chunk ^ swizzle(row);
            offset[j] = row * ld + c * 16;
            if (LAY == LAY_MN && c * 16 >= width) offset[j] = OUT_OF_RANGE;
        }
    }
    static __device__ inline int swizzle(int row) { return LAY == LAY_K ? swizzle_k<SPAN>(row) : swizzle_mn<B>(row); }
    __device__ inline u32x4_t desc() const {
        if (LAY == LAY_K) return make_desc(base, rows > 0 && width > 0 ? (rows - 1) * (int)ld + width : 0);
        return make_desc(base, rows > 0 && width > 0 ? (min(rows, SPAN / 2) - 1) * (int)ld + width : 0);
    }
    __device__ inline void stop() { rows = 0; }  // later stages read zeros
    template <bool NT = false> __device__ inline void issue(const u32x4_t& d, uint32_t to, int j, int wave) const { load_to_lds<NT>(to + (wave * NL + j) * 1024, offset[j], d); }
    __device__ inline void next(int stages = 1) {
        base += step * stages;
        if (LAY == LAY_K) width -= SPAN * stages;
        else rows -= SPAN / 2 * stages;
    }
    // before the last K step, of a row that may end inside it
    __device__ inline void cut(int wave) {
        if (LAY == LAY_K && width < SPAN) {
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const int p = (wave * NL + j) * 1024 + (threadIdx.x & 63) * 16;
                const int c = ((p % ROW) / 16) ^ swizzle(p / ROW);
                if (c * 16 >= width) offset[j] = OUT_OF_RANGE;
            }
        }
    }
};

// Reads of one operand's fragments (16 rows or columns by the values of one matrix instruction).
template <int FMT, int LAY, int B, int SPAN = 128> struct Reader {
    uint32_t at[2];   // LAY_K: lane address for the first and second half of a K step
    uint32_t cl, ch;  // LAY_MN: lane address without its column chunk; the chunk of fragment 0 before the swizzle
    uint32_t sw;

    __device__ inline void init(int first) {  // first row or column of the wave's part
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        if (LAY == LAY_K) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // 4-bit values: a lane's two blocks of 32 are neighbours, in both operands alike
                const int c = FMT == FMT_MX4 ? 2 * q + h : 4 * h + q;
                at[h] = (first + i) * SPAN + ((c ^ swizzle_k<SPAN>(i)) * 16);
            }
        } else {
            cl = (8 * q + (i >> 2)) * (2 * B) + (i & 1) * 8;
            ch = first / 8 + ((i & 3) >> 1);
            sw = swizzle_mn<B>(8 * q + (i >> 2));
        }
    }
    template <int F, int H> __device__ inline s16x8_t get(const char* tile) const {
        if (LAY == LAY_K) return *(const s16x8_t*)(tile + at[H] + F * 16 * SPAN);
        const uint32_t o = cl + (((ch + 2 * F) ^ sw) * 16);
        typedef __attribute__((address_space(3))) s16x4_t lds4;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + o + H * 64 * B));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + o + H * 64 * B + 8 * B));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

template <int I> struct Int { static constexpr int value = I; };
template <int N, typename F> static __device__ inline void repeat(F&& f) {
    if constexpr (N > 0) {
        repeat<N - 1>(f);
        f(Int<N - 1>{});
    }
}

static __device__ inline uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t v = {(__bf16)lo, (__bf16)hi};  // to nearest even
    return __builtin_bit_cast(uint32_t, v);
}

// One matrix instruction on fragments of 16 columns (b) and 16 rows (a); 4-bit ones take their blocks' scales from byte
// SB of sb and byte SA of sa.
template <int FMT, int SB, int SA> static __device__ inline f32x4_t multiply(const s16x8_t& b, const s16x8_t& a, f32x4_t c, int sb, int sa) {
    if constexpr (FMT == FMT_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, b), __builtin_bit_cast(bf16x8_t, a), c, 0, 0, 0);
    typedef int i32x4_t __attribute__((ext_vector_type(4)));
    const i32x4_t x = __builtin_bit_cast(i32x4_t, b), y = __builtin_bit_cast(i32x4_t, a);
    const i32x8_t u = {x[0], x[1], x[2], x[3], 0, 0, 0, 0}, v = {y[0], y[1], y[2], y[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, c, 4, 4, SB, sb, SA, sa);
}

// Where a wave's fragments go: a buffer that ends with the last column of the last row that exists, so that rows behind it and
// columns that are given an offset behind it are not stored, without a branch and with one address register (addresses of 64 bits
// were spilled, and every reload waited for the stores before it: gradient of 128 experts' weights 666 -> 645 us, of 16 experts',
// 8544 x 5888, 382 -> 344).
struct Sink {
    __amdgpu_buffer_rsrc_t to;
    uint32_t ld;  // bytes between rows
    uint32_t end; // bytes of a row that exist

    __device__ inline Sink(void* c, int64_t ldc, int esize, int rows, int cols) {
        ld = __builtin_amdgcn_readfirstlane((uint32_t)ldc * esize);
        asm volatile("" : "+s"(ld));  // places are formed where they are used: the compiler would keep them through the tiles
        end = (uint32_t)max(cols, 0) * esize;
        to = __builtin_amdgcn_make_buffer_rsrc(c, 0, __builtin_amdgcn_readfirstlane(rows > 0 && cols > 0 ? (rows - 1) * (int)ld + (int)end : 0), 0x27000);
    }
    // 16 bytes at byte `at` of row `row`; AUX: 2 is the non-temporal hint
    template <int AUX> __device__ inline void put(const u32x4_t& v, uint32_t row, uint32_t at) const {
        __builtin_amdgcn_raw_buffer_store_b128(v, to, at < end ? row * ld + at : OUT_OF_RANGE, 0, AUX);
    }
    template <int AUX> __device__ inline void add(const f32x4_t& v, uint32_t row, uint32_t at) const {
        const uint32_t place = at < end ? row * ld + at : OUT_OF_RANGE;
        const f32x4_t old = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(to, place, 0, 0));
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, old + v), to, place, 0, AUX);
    }
};

// Stores a wave's FM x FN fragments.  The weights are the first operand of the matrix instruction, so a lane has 4
// neighbouring columns of one row; two fragments change halves between neighbouring rows of 16 lanes, and every lane
// then stores 8 bf16 columns (16 bytes) of one row.
template <int OUT, int FM, int FN, int FAR>
static __device__ inline void store_tile(const f32x4_t (&acc)[FM][FN], const Sink& to) {
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    repeat<FM>([&](auto mf) {
        const int row = mf.value / (FM / 2) * FAR + mf.value % (FM / 2) * 16 + i;
        if constexpr (OUT == OUT_BF16) {
            repeat<FN / 2>([&](auto p) {
                const f32x4_t u = acc[mf.value][2 * p.value], v = acc[mf.value][2 * p.value + 1];
                const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(u[0], u[1]), pack_bf16(v[0], v[1]), false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(u[2], u[3]), pack_bf16(v[2], v[3]), false, false);
                to.put<0>(u32x4_t{lo[0], hi[0], lo[1], hi[1]}, row, p.value * 64 + (q & 1) * 32 + (q >> 1) * 16);
            });
        } else {
            repeat<FN>([&](auto nf) { to.put<0>(__builtin_bit_cast(u32x4_t, acc[mf.value][nf.value]), row, nf.value * 64 + q * 16); });
        }
    });
}

// The same for gradients of weights, which are the largest outputs and not read again soon: stores of whole 128-byte lines, with the
// non-temporal hint where AUX says so (with bands of 8: 32 experts, 2048 x 7168 from 5003 rows: 464 -> 415 us; with the hint on stores of
// 64 bytes 128 experts, 2048 x 1536 from 65528 rows take 868 us instead of 721).  Lanes 0 - 7 and 8 - 15 of every 16 change
// places, so that two stores of 16 rows by 64 bytes become two of 8 rows by 128.
template <int OUT, int FM, int FN, int FAR, int AUX>
static __device__ inline void store_lines(const f32x4_t (&acc)[FM][FN], const Sink& to) {
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    const bool low = i < 8;
    auto turn = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false); };  // from lane i ^ 8 of the 16
    repeat<FM>([&](auto mf) {
        const int row0 = mf.value / (FM / 2) * FAR + mf.value % (FM / 2) * 16 + (i & 7);
        repeat<FN * 16 * (OUT == OUT_BF16 ? 2 : 4) / 128>([&](auto p) {
            u32x4_t piece[2];  // of 64 bytes a row
            repeat<2>([&](auto h) {
                if constexpr (OUT == OUT_BF16) {
                    constexpr int N = 4 * p.value + 2 * h.value;
                    const f32x4_t u = acc[mf.value][N], v = acc[mf.value][N + 1];
                    const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(u[0], u[1]), pack_bf16(v[0], v[1]), false, false);
                    const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(u[2], u[3]), pack_bf16(v[2], v[3]), false, false);
                    piece[h.value] = u32x4_t{lo[0], hi[0], lo[1], hi[1]};
                } else {
                    piece[h.value] = __builtin_bit_cast(u32x4_t, acc[mf.value][2 * p.value + h.value]);
                }
            });
            u32x4_t a, b;  // rows 0 - 7 and 8 - 15 of the fragment
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t other = turn(low ? piece[1][w] : piece[0][w]);
                a[w] = low ? piece[0][w] : other;
                b[w] = low ? other : piece[1][w];
            }
            const uint32_t at = p.value * 128 + (low ? 0 : 64) + (OUT == OUT_BF16 ? (q & 1) * 32 + (q >> 1) * 16 : q * 16);
            repeat<2>([&](auto h) {
                if constexpr (OUT == OUT_F32_ADD) to.add<AUX>(__builtin_bit_cast(f32x4_t, h.value ? b : a), row0 + 8 * h.value, at);
                else to.put<AUX>(h.value ? b : a, row0 + 8 * h.value, at);
            });
            __builtin_amdgcn_sched_barrier(0);  // (fragments are turned one by one: there are no registers for more)
        });
    });
}

// Persistent: a workgroup goes through its tiles as one stream of K steps.  The stages of the next tile's first two steps are
// asked for during the last two of this one, so only the first tile waits for memory, and a tile's stores leave under the next one's
// products.
//
// Why 256 x 256: a K step of it is 64 KB for 8.4 MFLOP (bf16), two stages fit LDS, sums and fragments the 256 registers a lane
// has at eight waves, and a compute unit asks its L2 for 43 bytes a nanosecond at the rate below; 128 x 128 needs twice that.
// What bounds it: one product of 8192^3 the power (1400 TFLOP/s forward, 1430 gradient of the rows, 1385 of the weights, 4-bit
// 4330; MFMA instructions alone sustain 1948).  Ragged rows on many experts the loads, of which the L2s fetch 1.3 to 2.1 times what
// there is, and the steps' barriers behind them: 8192 rows, 14336 to 4096, two of 8 experts leading 831 us = 1160 TFLOP/s (with its last
// round whole 920; matrix pipes busy 65 % of the time), the gradient of 65536 rows of 128 experts, 1536 to 2048, 425 us = 970
// TFLOP/s (56 %), 4-bit 8192 rows, 4096 to 28672, 545 us = 3530 TFLOP/s (45 %; its 0.47 GB of results alone take 92 us).  The gradient of
// 128 experts' weights, 2048 x 1536 in fp32 from 65528 rows, memory: 617 us for 0.74 GB read and 1.61 GB written = 3.8 TB/s.
template <int FMT, int LA, int LB, int OUT, int BM, int BN, int WM, int WN, bool TAIL, bool LINES>
__global__ __launch_bounds__(WM * WN * 64) void grouped_tile_kernel(GroupedArgs g) {
    constexpr int NW = WM * WN, FH = BM / WM / 32, FN = BN / WN / 16, NLA = BM / 16 / NW, NLB = BN / 8 / NW;
    constexpr bool WEIGHTS = LA == LAY_MN, MX = FMT == FMT_MX4, CUT = BM < 256 || TAIL;
    constexpr int HALF = BM / 2, GROUP = HALF / WM;  // a wave has GROUP rows of each half of the tile: rows that are missing spare every wave alike
    constexpr int NS = (BM + BN) / 64 / NW;          // loads of scales a wave, every second K step
    constexpr int PER = MX ? 2 : 1;                  // K steps a load of scales is for
    static_assert(!MX || NS * 64 * NW == BM + BN, "scale loads");
    __shared__ __attribute__((aligned(1024))) char lds_a[2][2][HALF * 128];  // [half of the rows][slot]
    __shared__ __attribute__((aligned(1024))) char lds_b[2][BN * 128];
    __shared__ __attribute__((aligned(1024))) char lds_s[MX ? 2 * (BM + BN) * 16 : 16];
    __shared__ TileList list;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mt = (g.M + BM - 1) / BM, nt = (g.N + BN - 1) / BN;
    if (wave == 0) make_list<WEIGHTS, BM, TAIL>(g, (WEIGHTS ? mt * nt : nt) * (BM < 256 ? g.splits : 1), &list);
    block_barrier();
    const int height = WEIGHTS ? BM : __builtin_amdgcn_readfirstlane(list.height);
    int at = __builtin_amdgcn_readfirstlane(list.begin) + (blockIdx.x >> 3);
    const int last = __builtin_amdgcn_readfirstlane(list.end);
    if (at >= last) return;

    // ---- the stages: a cursor that runs two steps ahead of the products
    Loader<LA, HALF, NLA> la[2];
    Loader<LB, BN, NLB> lb;
    GroupedTile lt;
    int ls = 0, lsteps = 0, lfrom = 0, lpair = 0;  // its tile, step in it, steps of it, step of the reduction it begins with; which half
                                                   // of lds_s the last scales went to
    auto start = [&](const GroupedTile& t) {
        const int mrows = t.rows, ncols = g.N - t.n0;
        const char* wb = g.b + t.e * g.b_expert;
        // steps [from, to) of the reduction; at least two are gone through, those that are not there read zeros
        const int red = WEIGHTS ? t.n * 2 : g.kbytes, all = (red + 127) / 128;  // (bytes, as if its values were contiguous)
        // (4-bit: whole pairs, which share a load of scales)
        const int pairs = (all + PER - 1) / PER;
        const int from = CUT ? (uint32_t)(pairs * t.split) / t.pieces * PER : 0, to = CUT ? min(all, (int)((uint32_t)(pairs * (t.split + 1)) / t.pieces * PER)) : all;
        const int kb = CUT ? min(red, to * 128) : red;
        repeat<2>([&](auto u) {
            constexpr int R = u.value * HALF;
            if constexpr (LA == LAY_K) la[u.value].init(g.a + (int64_t)(t.lo + t.m0 + R) * g.lda, g.lda, mrows - R, kb, wave);
            else la[u.value].init(g.a + (int64_t)t.lo * g.lda + (int64_t)(t.m0 + R) * 2, g.lda, mrows - R, kb / 2, wave);
        });
        if constexpr (LB == LAY_K) lb.init(wb + (int64_t)t.n0 * g.ldb, g.ldb, ncols, kb, wave);
        else lb.init(WEIGHTS ? g.b + (int64_t)t.lo * g.ldb + (int64_t)t.n0 * 2 : wb + (int64_t)t.n0 * 2, g.ldb, ncols, kb / 2, wave);
        if constexpr (CUT) {
            la[0].next(from);
            la[1].next(from);
            lb.next(from);
        }
        lt = t;
        ls = 0;
        if constexpr (CUT) lfrom = from;
        lsteps = max(2, to - from);
    };
    // The loads of a stage in two parts, 0: upper rows, columns and scales; 1: lower rows.  begin(part), load_scales(), load(part, slot, 0 ..),
    // end(part).
    u32x4_t da[2], db;
    auto begin = [&](auto part) {
        if (LA == LAY_K) la[part.value].cut(wave);
        da[part.value] = la[part.value].desc();
        if constexpr (part.value == 0) {
            if (LB == LAY_K) lb.cut(wave);
            db = lb.desc();
        }
    };
    auto load_scales = [&]() {
        if ((ls & 1) == 0) {
            lpair ^= 1;
            const int mrows = lt.rows, ncols = g.N - lt.n0;
            repeat<NS>([&](auto j) {
                const int rows64 = wave * NS + j.value;  // 64 rows of a, or of b behind them
                const bool of_b = rows64 * 64 >= BM;
                const int row = rows64 * 64 - (of_b ? BM : 0), have = min((of_b ? ncols : mrows) - row, 64);
                const uint8_t* p = of_b ? g.sb + ((int64_t)lt.e * g.N + lt.n0 + row) * g.scale_ld : g.sa + (int64_t)(lt.lo + lt.m0 + row) * g.scale_ld;
                const u32x4_t d = make_desc((const char*)p + (lfrom + ls) * 8, have > 0 && (lfrom + ls) * 8 < g.scale_ld ? (have - 1) * g.scale_ld + 16 : 0);
                load_to_lds(lds_addr(lds_s) + lpair * (BM + BN) * 16 + rows64 * 1024, (threadIdx.x & 63) * g.scale_ld, d);
            });
        }
    };
    auto load = [&](auto part, int slot, auto j) {
        if constexpr (j.value < NLA) la[part.value].issue(da[part.value], lds_addr(lds_a[part.value][0]) + slot * HALF * 128, j.value, wave);
        else lb.issue(db, lds_addr(lds_b[0]) + slot * BN * 128, j.value - NLA, wave);
    };
    auto end = [&](auto part) {
        la[part.value].next();
        if constexpr (part.value == 0) lb.next();
        else ++ls;
    };

    f32x4_t acc[2 * FH][FN];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < 2 * FH; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    const int wm = wave / WN, wn = wave % WN;
    Reader<FMT, LA, HALF> ra;
    Reader<FMT, LB, BN> rb;
    ra.init(wm * GROUP);
    rb.init(wn * FN * 16);

    // A K step is four phases of FH x FN products: (upper rows, first half of the reduction), (upper, second), (lower, first),
    // (lower, second).  The fragments of a phase are read during the one before it, those of the columns once for both halves of the
    // rows.  So the upper rows and the columns of a stage are free before phase 1 and the lower rows before phase 3; the stage after
    // next is asked for there (three loads a wave and phase, what the compute unit's one memory pipe takes meanwhile) and has a step and
    // a quarter to arrive.
    s16x8_t fa[2][FH], fb[2][FN];
    int sa[FH], sb[FN / 2];  // scale bytes of two fragments each: (first half, second half) of both
    int slot = 0, pair = 1;  // of the step at hand: its slot in lds_a and lds_b, its half of lds_s
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    auto read_scale = [&](auto i, int pr, int odd) {  // pair i of the wave's rows, then of its columns
        constexpr int I = i.value, ROW = 2 * I / FH * HALF + 2 * I % FH * 16;
        const char* ts = lds_s + pr * (BM + BN) * 16 + odd * 8 + ((threadIdx.x >> 4) & 3) * 2 + (threadIdx.x & 15) * 16;
        const uint16_t* r = (const uint16_t*)(I < FH ? ts + (wm * GROUP + ROW) * 16 : ts + BM * 16 + (wn * FN + 2 * (I - FH)) * 256);
        return __builtin_bit_cast(int, u16x2_t{r[0], r[128]});
    };
    int live = 2;  // halves in which this wave has rows
    auto phase = [&](auto p, int odd) {  // odd: of the next step, in its tile
        constexpr int P = p.value, U = P >> 1, H = P & 1, NP = (P + 1) & 3, NU = NP >> 1, NH = NP & 1;
        constexpr bool NEWB = NP < 2;  // the next phase's columns are read as well
        constexpr int READS = FH + (NEWB ? FN : 0), PROD = FH * FN, ALL = NLA + NLB;
        constexpr int PART = P == 3, FIRST = P == 2 ? ALL / 2 : 0, NL = P == 1 ? ALL / 2 : P == 2 ? ALL - ALL / 2 : P == 3 ? NLA : 0;
        const int from = P == 3 ? slot ^ 1 : slot;
        const char* ta = lds_a[NU][0] + from * HALF * 128;
        const char* tb = lds_b[0] + from * BN * 128;
        int na[FH], nb[FN / 2];
        if constexpr (H == 1) {
            wait_loads<2 * NLA + NLB>();
            block_barrier();
            if constexpr (MX && P == 1) load_scales();
            if (MX && P == 3 && !odd) pair ^= 1;
        }
        // what goes on beside product I: the next phase's fragments in the first places, the columns' before the rows' as the
        // products need them; the loads of a stage; the next step's scales
        auto beside = [&](auto i) {
            constexpr int I = i.value;
            if constexpr (I < READS) {
                if constexpr (I < READS - FH) fb[NH][I] = rb.template get<I, NH>(tb);
                else fa[NH][I - (READS - FH)] = ra.template get<I - (READS - FH), NH>(ta);
            }
            if constexpr (NL > 0) repeat<(I + 1) * NL / PROD - I * NL / PROD>([&](auto j) { load(Int<PART>{}, slot, Int<FIRST + I * NL / PROD + j.value>{}); });
            if constexpr (H == 0 && I == PROD / 2) begin(Int<U>{});  // what the next phase asks for
            if constexpr (P == 3 && MX) {
                constexpr int NSC = FH + FN / 2, s0 = I * NSC / PROD, s1 = (I + 1) * NSC / PROD;
                if constexpr (s1 > s0) {
                    if constexpr (s0 < FH) na[s0] = read_scale(Int<s0>{}, pair, odd);
                    else nb[s0 - FH] = read_scale(Int<s0>{}, pair, odd);
                }
            }
        };
        if (live > U) {
            repeat<PROD>([&](auto i) {
                // columns there and back: consecutive products share an operand (what does not toggle costs no power, and power bounds the clock)
                constexpr int m = i.value / FN, n = m & 1 ? FN - 1 - i.value % FN : i.value % FN, M = U * FH + m;
                acc[M][n] = multiply<FMT, H + 2 * (n & 1), H + 2 * (M & 1)>(fb[H][n], fa[H][m], acc[M][n], sb[n / 2], sa[M / 2]);
                beside(i);
                __builtin_amdgcn_sched_barrier(0);
            });
        } else {
            repeat<PROD>(beside);
        }
        if constexpr (P >= 2) end(Int<P - 2>{});
        if constexpr (P == 3) {
            if constexpr (MX) {
                repeat<FH>([&](auto f) { sa[f.value] = na[f.value]; });
                repeat<FN / 2>([&](auto f) { sb[f.value] = nb[f.value]; });
            }
            slot ^= 1;
        }
    };

    start(find_tile<WEIGHTS, BM, BN, TAIL>(g, list, BM < 256 ? g.splits : 1, WEIGHTS ? BM : height, mt, nt, at));
    repeat<2>([&](auto s) {
        repeat<2>([&](auto part) {
            begin(part);
            if constexpr (MX && part.value == 0) load_scales();
            repeat<NLA + (part.value == 0 ? NLB : 0)>([&](auto j) { load(part, s.value, j); });
            end(part);
        });
    });
    clear();
    wait_loads<3 * NLA + NLB>();
    block_barrier();
    if constexpr (MX) {
        repeat<FH>([&](auto f) { sa[f.value] = read_scale(f, 1, 0); });
        repeat<FN / 2>([&](auto f) { sb[f.value] = read_scale(Int<FH + f.value>{}, 1, 0); });
    }
    repeat<FN>([&](auto f) { fb[0][f.value] = rb.template get<f.value, 0>(lds_b[0]); });
    repeat<FH>([&](auto f) { fa[0][f.value] = ra.template get<f.value, 0>(lds_a[0][0]); });
    for (;;) {
        const GroupedTile t = lt;
        const int mrows = t.rows;
        live = (mrows > wm * GROUP) + (mrows > HALF + wm * GROUP);
        int left = lsteps;
        for (int kt = 0; left > 0; ++kt, --left) {
            asm volatile("" : "+s"(left));  // one loop body: the compiler would peel the last steps
            if (left == 2) {                // from here on the loads are the next tile's
                at += gridDim.x >> 3;
                if (at < last) {
                    start(find_tile<WEIGHTS, BM, BN, TAIL>(g, list, BM < 256 ? g.splits : 1, WEIGHTS ? BM : height, mt, nt, at));
                } else {
                    la[0].stop();
                    la[1].stop();
                    lb.stop();
                    ls = 1;  // (one more pair of scales is asked for at the most, of this tile, which nobody reads)
                }
            }
            const int odd = left == 1 ? 0 : (kt + 1) & 1;
            repeat<4>([&](auto p) { phase(p, odd); });
        }
        const int m = t.m0 + wm * GROUP, n = t.n0 + wn * FN * 16;
        const int64_t row = WEIGHTS ? (int64_t)t.e * g.M + m : (int64_t)t.lo + m;
        constexpr int esize = OUT == OUT_BF16 ? 2 : 4;
        if (CUT && t.pieces > 1) {
            // the ranges of whole products leave slabs like c, those of the last tiles (a workgroup has one at the most, its last) slots
            float* to = BM < 256 ? g.part + t.split * g.slab + row * g.N + n
                                 : g.part + ((blockIdx.x & 7) * SIDE + (blockIdx.x >> 3)) * PIECE + wm * GROUP * 256 + wn * FN * 16;
            store_tile<OUT_F32, 2 * FH, FN, HALF>(acc, Sink(to, BM < 256 ? g.N : 256, 4, mrows - wm * GROUP, g.N - n));
        } else if (!(OUT == OUT_F32_ADD && t.n == 0)) {
            const Sink to((char*)g.c + (row * g.ldc + n) * esize, g.ldc, esize, mrows - wm * GROUP, g.N - n);
            if constexpr (!WEIGHTS) store_tile<OUT, 2 * FH, FN, HALF>(acc, to);
            else store_lines<OUT, 2 * FH, FN, HALF, LINES ? 2 : 0>(acc, to);
        }
        if (at >= last) break;
        clear();
    }
    wait_loads<0>();  // nothing may arrive in LDS after the workgroup has left it
}

// One workgroup a compute unit (two where two fit), in eights so that every XCD has as many.
template <int FMT, int LA, int LB, int OUT, int BM, int BN, int WM, int WN, bool TAIL = false, bool LINES = false> static inline hipError_t launch_tiles(const GroupedArgs& g, hipStream_t st) {
    constexpr int blocks = BM * BN > 128 * 128 ? 256 : 512;
    grouped_tile_kernel<FMT, LA, LB, OUT, BM, BN, WM, WN, TAIL, LINES><<<blocks, WM * WN * 64, 0, st>>>(g);
    return hipGetLastError();
}

// The kernels' units: a product of g on tiles of bm rows.
hipError_t grouped_launch_row_major(const GroupedArgs& g, int bm, hipStream_t st);
hipError_t grouped_launch_transposed(const GroupedArgs& g, int bm, hipStream_t st);
hipError_t grouped_launch_mx(const GroupedArgs& g, int bm, hipStream_t st);
hipError_t grouped_launch_weights(const GroupedArgs& g, int out, int bm, hipStream_t st);
