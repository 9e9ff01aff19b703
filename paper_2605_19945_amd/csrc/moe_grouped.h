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
};

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;  // an offset behind the end of every descriptor (those are below 2 GB)

static __device__ inline uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(const lds_char*)p; }

static __device__ inline u32x4_t make_desc(const char* base, uint32_t bytes) {
    const uint64_t p = (uint64_t)base;
    u32x4_t d;
    d[0] = __builtin_amdgcn_readfirstlane((uint32_t)p);
    d[1] = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32) & 0xffffu);
    d[2] = __builtin_amdgcn_readfirstlane(bytes);
    d[3] = 0x00027000u;
    return d;
}

// 16 bytes a lane from memory to LDS at `to` + 16 * lane.  Inline asm, so that the compiler does not wait for it at the
// next LDS read; it has no output registers.
static __device__ inline void load_to_lds(uint32_t to, uint32_t offset, const u32x4_t& desc) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(desc) : "memory");
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
};

// Inside one expert's mt x nt tiles: bands of up to 8 row tiles, row tiles fastest, so that the 32 compute units of an XCD
// work on about 8 x 4 neighbouring tiles and share their panels in its L2.
static __device__ inline void place_in_band(int t, int mt, int nt, int* m, int* n) {
    const int band = t / (8 * nt), r = t - band * 8 * nt;
    const int h = min(8, mt - 8 * band);
    *n = r / h;
    *m = 8 * band + r - *n * h;
}

// The tile of workgroup `bid` of a product over ragged rows: each XCD (bid % 8) takes one stretch of the list of all
// tiles, which follows from the offsets alone; every wave finds its entry by itself (4 experts a lane).  False: no tile.
template <int BM> static __device__ inline bool find_row_tile(const GroupedArgs& g, int nt, int bid, int bn, GroupedTile* out) {
    const int lane = threadIdx.x & 63;
    int cnt[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = 4 * lane + j;
        int lo = 0, n = 0;
        if (e < g.E) expert_rows(g.offsets, e, g.rows_cap, &lo, &n);
        cnt[j] = (n + BM - 1) / BM;
        sum += cnt[j];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    const int mts = __builtin_amdgcn_readlane(incl, 63);
    const int64_t total = (int64_t)mts * nt;
    const int xcd = bid & 7, idx = bid >> 3;
    const int64_t base = total >> 3, rem = total & 7;
    if (idx >= base + (xcd < rem ? 1 : 0)) return false;
    const int64_t t = xcd * base + (xcd < rem ? xcd : rem) + idx;
    const int tm = (int)(t / nt);  // row tiles of earlier experts are all of theirs times nt
    const uint64_t past = __ballot(incl > tm);
    if (past == 0) return false;
    const int src = __builtin_ctzll(past);
    int before = __builtin_amdgcn_readlane(incl - sum, src), e = 4 * src, mt = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = __builtin_amdgcn_readlane(cnt[j], src);
        if (mt == 0) {
            if (tm < before + c) {
                mt = c;
                e = 4 * src + j;
            } else {
                before += c;
            }
        }
    }
    int m, n;
    place_in_band((int)(t - (int64_t)before * nt), mt, nt, &m, &n);
    out->e = e;
    expert_rows(g.offsets, e, g.rows_cap, &out->lo, &out->n);
    out->lo = __builtin_amdgcn_readfirstlane(out->lo);
    out->n = __builtin_amdgcn_readfirstlane(out->n);
    out->m0 = m * BM;
    out->n0 = n * bn;
    return true;
}

// The tile of workgroup `bid` of a weight gradient: every expert has mt x nt tiles, and each XCD takes an eighth of
// every expert's, because an expert's tiles cost what it has rows.
static __device__ inline bool find_weight_tile(const GroupedArgs& g, int mt, int nt, int bid, int bm, int bn, GroupedTile* out) {
    const int per = mt * nt, px = (per + 7) / 8, xcd = bid & 7, idx = bid >> 3;
    const int e = idx / px, t = xcd * px + idx % px;
    if (e >= g.E || t >= per) return false;
    int m, n;
    place_in_band(t, mt, nt, &m, &n);
    out->e = e;
    expert_rows(g.offsets, e, g.rows_cap, &out->lo, &out->n);
    out->lo = __builtin_amdgcn_readfirstlane(out->lo);
    out->n = __builtin_amdgcn_readfirstlane(out->n);
    out->m0 = m * bm;
    out->n0 = n * bn;
    return true;
}

// 16-byte chunk c of a row lies at chunk c ^ swizzle(row) of its LDS row, so that the lanes that read together fall on
// different banks.  LAY_MN: rows 0-3 and 8-11, two neighbouring chunks.  LAY_K: a 16-byte read serves lanes 0-3, 12-15 and 20-27 together,
// so rows 0-3 and 12-15 of one chunk (swizzles 0 to 3) and rows 4-11 of a second one (4 to 7): whichever two chunks of an even distance
// below 4 or neighbouring ones those are, the two sets stay apart (no conflicts counted for either format).
static __device__ inline int swizzle_k(int row) {
    const int t = row >> 1;
    return (t & 1) | (t >> 1 & 2) | ((t ^ t << 1) & 4);
}

// One operand's share of a wave: NL loads of 1 KiB a K step.
template <int LAY, int B, int NL> struct Loader {
    static constexpr int ROW = LAY == LAY_K ? 128 : 2 * B;  // bytes of a row in LDS
    const char* base;
    int64_t step;        // bytes to the next K step
    uint32_t ld, width;  // bytes between rows; bytes of the last row that belong to the operand
    int rows;            // LAY_K: valid rows of the tile; LAY_MN: rows (k) left from this step on
    uint32_t offset[NL];

    // `first`: the address of the tile's first value; `valid`: rows (LAY_K) or columns (LAY_MN) of the tile that exist;
    // `k`: bytes (LAY_K) or rows (LAY_MN) of the reduction
    __device__ inline void init(const char* first, int64_t ld_, int valid, int k, int wave) {
        const int lane = threadIdx.x & 63;
        base = first;
        ld = (uint32_t)ld_;
        if (LAY == LAY_K) {
            step = 128;
            rows = min(valid, B);
            width = k;
        } else {
            step = 64 * ld_;
            rows = k;
            width = 2 * min(valid, B);
        }
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int p = (wave * NL + j) * 1024 + lane * 16;
            const int row = p / ROW, chunk = (p % ROW) / 16;
            const int c = chunk ^ swizzle(row);
            offset[j] = row * ld + c * 16;
            if (LAY == LAY_MN && c * 16 >= (int)width) offset[j] = OUT_OF_RANGE;
        }
    }
    static __device__ inline int swizzle(int row) { return LAY == LAY_K ? swizzle_k(row) : 2 * ((row & 3) + 4 * ((row >> 3) & 1)); }
    __device__ inline u32x4_t desc() const {
        if (LAY == LAY_K) return make_desc(base, rows > 0 ? (rows - 1) * ld + width : 0);
        return make_desc(base, rows > 0 ? (min(rows, 64) - 1) * ld + width : 0);
    }
    __device__ inline void issue(const u32x4_t& d, uint32_t to, int j, int wave) const { load_to_lds(to + (wave * NL + j) * 1024, offset[j], d); }
    __device__ inline void next() {
        base += step;
        if (LAY == LAY_K) width -= 128;
        else rows -= 64;
    }
    // before the last K step, of a row that may end inside it
    __device__ inline void cut(int wave) {
        if (LAY == LAY_K && width < 128) {
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const int p = (wave * NL + j) * 1024 + (threadIdx.x & 63) * 16;
                const int c = ((p % ROW) / 16) ^ swizzle(p / ROW);
                if (c * 16 >= (int)width) offset[j] = OUT_OF_RANGE;
            }
        }
    }
};

// Reads of one operand's fragments (16 rows or columns by the values of one matrix instruction).
template <int FMT, int LAY, int B> struct Reader {
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
                at[h] = (first + i) * 128 + ((c ^ swizzle_k(i)) * 16);
            }
        } else {
            cl = (8 * q + (i >> 2)) * (2 * B) + (i & 1) * 8;
            ch = first / 8 + ((i & 3) >> 1);
            sw = 2 * ((i >> 2) + 4 * (q & 1));
        }
    }
    template <int F, int H> __device__ inline s16x8_t get(const char* tile) const {
        if (LAY == LAY_K) return *(const s16x8_t*)(tile + at[H] + F * 2048);
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

// Stores a wave's FM x FN fragments.  The weights are the first operand of the matrix instruction, so a lane has 4
// neighbouring columns of one row; two fragments change halves between neighbouring rows of 16 lanes, and every lane
// then stores 8 bf16 columns (16 bytes) of one row.
template <int OUT, int FM, int FN>
static __device__ inline void store_tile(const f32x4_t (&acc)[FM][FN], void* c, int64_t ldc, int rows, int cols) {
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    repeat<FM>([&](auto mf) {
        const int row = mf.value * 16 + i;
        if constexpr (OUT == OUT_BF16) {
            repeat<FN / 2>([&](auto p) {
                const f32x4_t u = acc[mf.value][2 * p.value], v = acc[mf.value][2 * p.value + 1];
                const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16(u[0], u[1]), pack_bf16(v[0], v[1]), false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16(u[2], u[3]), pack_bf16(v[2], v[3]), false, false);
                const int col = (2 * p.value + (q & 1)) * 16 + (q >> 1) * 8;
                if (row < rows && col < cols) {
                    const u32x4_t w = {lo[0], hi[0], lo[1], hi[1]};
                    *(u32x4_t*)((uint16_t*)c + row * ldc + col) = w;
                }
            });
        } else {
            repeat<FN>([&](auto nf) {
                const int col = nf.value * 16 + q * 4;
                if (row < rows && col < cols) {
                    f32x4_t* to = (f32x4_t*)((float*)c + row * ldc + col);
                    f32x4_t v = acc[mf.value][nf.value];
                    if (OUT == OUT_F32_ADD) v += *to;
                    *to = v;
                }
            });
        }
    });
}

template <int FMT, int LA, int LB, int OUT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void grouped_tile_kernel(GroupedArgs g) {
    constexpr int NW = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16, NLA = BM / 8 / NW, NLB = BN / 8 / NW;
    constexpr bool WEIGHTS = LA == LAY_MN, MX = FMT == FMT_MX4;
    constexpr int NS = (BM + BN) / 64 / NW;  // loads of scales a wave, every second K step
    static_assert(!MX || NS * 64 * NW == BM + BN, "scale loads");
    __shared__ __attribute__((aligned(1024))) char lds_a[2 * BM * 128];
    __shared__ __attribute__((aligned(1024))) char lds_b[2 * BN * 128];
    __shared__ __attribute__((aligned(1024))) char lds_s[MX ? 2 * (BM + BN) * 16 : 16];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    GroupedTile t;
    if (WEIGHTS ? !find_weight_tile(g, (g.M + BM - 1) / BM, (g.N + BN - 1) / BN, blockIdx.x, BM, BN, &t)
                : !find_row_tile<BM>(g, (g.N + BN - 1) / BN, blockIdx.x, BN, &t))
        return;
    const int mrows = WEIGHTS ? g.M - t.m0 : t.n - t.m0, ncols = g.N - t.n0;
    if (OUT == OUT_F32_ADD && t.n == 0) return;

    Loader<LA, BM, NLA> la;
    Loader<LB, BN, NLB> lb;
    const char* wb = g.b + t.e * g.b_expert;
    const int red = LA == LAY_K ? g.kbytes / (MX ? 1 : 2) : t.n;  // reduction: values (bytes of 4-bit values)
    if constexpr (LA == LAY_K) la.init(g.a + (int64_t)(t.lo + t.m0) * g.lda, g.lda, mrows, g.kbytes, wave);
    else la.init(g.a + (int64_t)t.lo * g.lda + (int64_t)t.m0 * 2, g.lda, mrows, red, wave);
    if constexpr (LB == LAY_K) lb.init(wb + (int64_t)t.n0 * g.ldb, g.ldb, ncols, g.kbytes, wave);
    else lb.init(WEIGHTS ? g.b + (int64_t)t.lo * g.ldb + (int64_t)t.n0 * 2 : wb + (int64_t)t.n0 * 2, g.ldb, ncols, red, wave);
    const int steps = (red + (MX ? 127 : 63)) / (MX ? 128 : 64);

    // The loads of a stage, one at a time: begin(kt), load(kt, 0 .. NLA + NLB - 1), end().
    u32x4_t da, db;
    auto begin = [&](int kt) {
        da = la.desc();
        db = lb.desc();
        if constexpr (MX) {
            if ((kt & 1) == 0) repeat<NS>([&](auto j) {
                const int part = wave * NS + j.value;  // 64 rows of a, or of b behind them
                const bool of_b = part * 64 >= BM;
                const int row = part * 64 - (of_b ? BM : 0), have = min((of_b ? ncols : mrows) - row, 64);
                const uint8_t* p = of_b ? g.sb + ((int64_t)t.e * g.N + t.n0 + row) * g.scale_ld : g.sa + (int64_t)(t.lo + t.m0 + row) * g.scale_ld;
                const u32x4_t d = make_desc((const char*)p + kt * 8, have > 0 ? (have - 1) * g.scale_ld + 16 : 0);
                load_to_lds(lds_addr(lds_s) + ((kt >> 1) & 1) * (BM + BN) * 16 + part * 1024, (threadIdx.x & 63) * g.scale_ld, d);
            });
        }
    };
    auto load = [&](int kt, auto j) {
        if constexpr (j.value < NLA) la.issue(da, lds_addr(lds_a) + (kt & 1) * BM * 128, j.value, wave);
        else lb.issue(db, lds_addr(lds_b) + (kt & 1) * BN * 128, j.value - NLA, wave);
    };
    auto cut = [&]() {
        la.cut(wave);
        lb.cut(wave);
    };
    auto issue = [&](int kt) {
        begin(kt);
        repeat<NLA + NLB>([&](auto j) { load(kt, j); });
        la.next();
        lb.next();
    };

    f32x4_t acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int wm = wave / WN, wn = wave % WN;
    Reader<FMT, LA, BM> ra;
    Reader<FMT, LB, BN> rb;
    ra.init(wm * FM * 16);
    rb.init(wn * FN * 16);

    // A K step is four phases of FM / 2 x FN products: (first half of the reduction, upper rows), (first, lower), (second,
    // upper), (second, lower).  The fragments of a phase are read during the one before it.  Before the last phase of a step the
    // next stage is published: by then every wave holds all it needs of this one, whose memory takes the stage after next.
    s16x8_t fa[2][FM / 2], fb[2][FN];
    int sa[FM / 2], sb[FN / 2];  // scale bytes of two fragments each: (first half, second half) of both
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    const char* ts0 = lds_s + ((threadIdx.x >> 4) & 3) * 2 + (threadIdx.x & 15) * 16;
    auto read_scale = [&](auto i, int kt) {  // pair i of the wave's rows, then of its columns
        const char* ts = ts0 + ((kt >> 1) & 1) * (BM + BN) * 16 + (kt & 1) * 8;
        const uint16_t* r = (const uint16_t*)(i.value < FM / 2 ? ts + (wm * FM + 2 * i.value) * 256 : ts + BM * 16 + (wn * FN + 2 * i.value - FM) * 256);
        return __builtin_bit_cast(int, u16x2_t{r[0], r[128]});
    };
    // WITH: the last phase of a step also asks for the stage after next.
    auto phase = [&](auto p, auto with, int kt) {
        constexpr int P = p.value, H = P >> 1, U = P & 1, NP = (P + 1) & 3, NH = NP >> 1, NU = NP & 1, NL = NLA + NLB;
        constexpr int READS = FM / 2 + (NU == 0 ? FN : 0), PROD = FM / 2 * FN;
        const int ns = (P == 3 ? kt + 1 : kt) & 1;
        const char* ta = lds_a + ns * BM * 128;
        const char* tb = lds_b + ns * BN * 128;
        int na[FM / 2], nb[FN / 2];
        if constexpr (P == 3) {
            wait_loads<0>();
            block_barrier();
            if constexpr (with.value) begin(kt + 2);
        }
        repeat<PROD>([&](auto i) {
            constexpr int I = i.value, m = I / FN, n = I % FN, M = U * FM / 2 + m;
            acc[M][n] = multiply<FMT, H + 2 * (n & 1), H + 2 * (M & 1)>(fb[H][n], fa[U][m], acc[M][n], sb[n / 2], sa[M / 2]);
            // the next phase's fragments in the first places, the columns' before the rows' as the products need them
            if constexpr (I < READS) {
                if constexpr (I < READS - FM / 2) fb[NH][I] = rb.template get<I, NH>(tb);
                else fa[NU][I - (READS - FM / 2)] = ra.template get<NU * FM / 2 + I - (READS - FM / 2), NH>(ta);
            }
            if constexpr (P == 3 && with.value) repeat<(I + 1) * NL / PROD - I * NL / PROD>([&](auto j) { load(kt + 2, Int<I * NL / PROD + j.value>{}); });
            if constexpr (P == 3 && MX) {
                constexpr int NSC = (FM + FN) / 2, s0 = I * NSC / PROD, s1 = (I + 1) * NSC / PROD;
                if constexpr (s1 > s0) {
                    if constexpr (s0 < FM / 2) na[s0] = read_scale(Int<s0>{}, kt + 1);
                    else nb[s0 - FM / 2] = read_scale(Int<s0>{}, kt + 1);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (P == 3) {
            if constexpr (with.value) {
                la.next();
                lb.next();
            }
            if constexpr (MX) {
                repeat<FM / 2>([&](auto f) { sa[f.value] = na[f.value]; });
                repeat<FN / 2>([&](auto f) { sb[f.value] = nb[f.value]; });
            }
        }
    };
    auto step = [&](auto with, int kt) {
        phase(Int<0>{}, with, kt);
        phase(Int<1>{}, with, kt);
        phase(Int<2>{}, with, kt);
        phase(Int<3>{}, with, kt);
    };
    if (steps > 0) {
        if (steps == 1) cut();
        issue(0);
        if (steps == 2) cut();
        wait_loads<0>();
        block_barrier();
        if (steps > 1) issue(1);
        if constexpr (MX) {
            repeat<FM / 2>([&](auto f) { sa[f.value] = read_scale(f, 0); });
            repeat<FN / 2>([&](auto f) { sb[f.value] = read_scale(Int<FM / 2 + f.value>{}, 0); });
        }
        repeat<FN>([&](auto f) { fb[0][f.value] = rb.template get<f.value, 0>(lds_b); });
        repeat<FM / 2>([&](auto f) { fa[0][f.value] = ra.template get<f.value, 0>(lds_a); });
        int kt = 0;
        for (; kt + 2 < steps; ++kt) {
            if (kt + 3 == steps) cut();
            step(Int<1>{}, kt);
        }
        for (; kt < steps; ++kt) step(Int<0>{}, kt);
    }

    const int m = t.m0 + wm * FM * 16, n = t.n0 + wn * FN * 16;
    const int64_t row = WEIGHTS ? (int64_t)t.e * g.M + m : (int64_t)t.lo + m;
    const int esize = OUT == OUT_BF16 ? 2 : 4;
    store_tile<OUT, FM, FN>(acc, (char*)g.c + (row * g.ldc + n) * esize, g.ldc, (WEIGHTS ? g.M : t.n) - m, g.N - n);
}
