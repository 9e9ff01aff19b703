// The products grouped by expert where an expert has few rows: the weights are read once and bound the time, so the work
// is cut for reads in flight instead of products.
//
// A tile is BM rows of an expert times 128 columns (row-major weights: a stage is 32 rows of 256 bytes) or 64 (transposed and 4-bit
// weights: 64 rows of 128 bytes).  The four waves of a workgroup split the reduction, stage by stage in turn, and each keeps a ring
// of its own in LDS with RING stages of 8 KiB of weights on their way; a stage's place is asked for again as soon as its
// fragments are in registers.  No wave waits for another before the end of a tile, where the partial sums are added in the order of the
// waves.  A workgroup (one a compute unit) goes through its tiles as one stream, so the ring stays full from tile to tile.
// Measured: two tokens on two experts, 4096 to 28672: 0.47 GB of weights in 79 us = 5.9 TB/s; 128 rows on 8 experts, the same
// widths in 4 bits: 0.50 GB in 87 us = 5.7 TB/s.  A kernel that only reads reaches 7.1 TB/s; the rest is the first stages' latency
// and the last tiles' unequal end.  Rings: what 160 KB of LDS hold beside the partial sums, three stages for 16 rows, two for 32.
#pragma once
#include "moe_grouped.h"

static __device__ inline void hold(s16x8_t& f) { asm volatile("" : "+v"(f)); }

template <int FMT, int LB, int BM, int RING> __global__ __launch_bounds__(256) void grouped_stream_kernel(GroupedArgs g) {
    constexpr bool MX = FMT == FMT_MX4;
    constexpr int NW = 4, BN = LB == LAY_MN ? 128 : 64, SPAN = LB == LAY_MN ? 64 : 128, HALVES = SPAN / 64, PER = MX ? 2 : 1;
    constexpr int FM = BM / 16, FN = BN / 16, XB = BM * SPAN, WB = 8192, NLX = XB / 1024, NLW = WB / 1024;
    constexpr int SB = MX ? 2 * (BM + BN) * 16 : 0, WAVE = RING * (XB + WB) + SB;
    __shared__ __attribute__((aligned(1024))) char lds[NW * WAVE];
    __shared__ __attribute__((aligned(16))) float parts[NW][BM * BN];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
    RowTiles<BM> tiles;
    tiles.init(g, (g.N + BN - 1) / BN, g.splits);
    int at = tiles.begin + (blockIdx.x >> 3);
    if (at >= tiles.end) return;

    // Turns of the waves (a stage each, 4-bit ones a pair that shares a load of scales), cut into the ranges of the reduction.  As many
    // stages for every wave and range, and enough that the loads are never two tiles ahead: the last ones may read zeros.
    constexpr int TURN = SPAN * PER * NW;
    const int turns = (g.kbytes + TURN - 1) / TURN;
    const int mine = max((turns + g.splits - 1) / g.splits, (RING + PER - 1) / PER) * PER;
    char* ring = lds + wave * WAVE;
    char* scales = ring + RING * (XB + WB);

    // ---- the cursor of the loads
    Loader<LAY_K, BM, NLX, SPAN> lx;
    Loader<LB, BN, NLW, SPAN> lw;
    GroupedTile lt;
    int ls = 0, lfrom = 0;            // its stage in the tile, the turn that begins with
    int place = 0, half = 0;          // its place in the ring, which half of the scales comes next
    auto start = [&]() {
        lt = tiles.find(at, BN, g.splits);
        lfrom = turns * lt.split / g.splits;
        const int kb = min(g.kbytes, turns * (lt.split + 1) / g.splits * TURN);
        lx.init(g.a + (int64_t)(lt.lo + lt.m0) * g.lda, g.lda, lt.n - lt.m0, kb, 0);
        const char* wb = g.b + lt.e * g.b_expert;
        if constexpr (LB == LAY_K) lw.init(wb + (int64_t)lt.n0 * g.ldb, g.ldb, g.N - lt.n0, kb, 0);
        else lw.init(wb + (int64_t)lt.n0 * 2, g.ldb, g.N - lt.n0, kb / 2, 0);
        lx.next((lfrom * NW + wave) * PER);
        lw.next((lfrom * NW + wave) * PER);
        ls = 0;
    };
    auto issue = [&]() {
        if (ls == mine) {
            at += gridDim.x >> 3;
            if (at < tiles.end) {
                start();
            } else {
                lx.stop();
                lw.stop();
                ls = -(1 << 30);  // (no scales either)
            }
        }
        lx.cut(0);
        lw.cut(0);
        const u32x4_t dx = lx.desc(), dw = lw.desc();
        const uint32_t to = lds_addr(ring) + place * (XB + WB);
        if constexpr (MX) {
            if ((ls & 1) == 0) {
                const int k = ((lfrom + (ls >> 1)) * NW + wave) * 16, left = ls >= 0 ? g.scale_ld - k : 0;
                const uint8_t* px = g.sa + (int64_t)(lt.lo + lt.m0) * g.scale_ld + k;
                const uint8_t* pw = g.sb + ((int64_t)lt.e * g.N + lt.n0) * g.scale_ld + k;
                const uint32_t there = lds_addr(scales) + half * (BM + BN) * 16;
                load_to_lds<true>(there + BM * 16, lane * g.scale_ld, make_desc((const char*)pw, left > 0 ? (min(g.N - lt.n0, BN) - 1) * g.scale_ld + 16 : 0));
                // rows of x in the first lanes; the others would land on the weights' scales
                if (lane < BM) load_to_lds(there, lane * g.scale_ld, make_desc((const char*)px, left > 0 ? (min(lt.n - lt.m0, BM) - 1) * g.scale_ld + 16 : 0));
                half ^= 1;
            }
        }
        repeat<NLX>([&](auto j) { lx.issue(dx, to, j.value, 0); });
        repeat<NLW>([&](auto j) { lw.template issue<true>(dw, to + XB, j.value, 0); });
        const int stages = MX && (ls & 1) == 0 ? 1 : (NW - 1) * PER + 1;
        lx.next(stages);
        lw.next(stages);
        ++ls;
        place = place == RING - 1 ? 0 : place + 1;
    };

    Reader<FMT, LAY_K, BM, SPAN> rx;
    Reader<FMT, LB, BN, SPAN> rw;
    rx.init(0);
    rw.init(0);
    start();
    GroupedTile t = lt;
    repeat<RING>([&](auto) { issue(); });
    int from = 0, have = 1;  // place of the stage at hand; half of its scales, turned at every first one of a pair
    for (;;) {
        f32x4_t acc[FM][FN];
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) acc[m][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        const int mrows = min(t.n - t.m0, BM), ncols = g.N - t.n0;
        GroupedTile next = t;
        bool more = true;
        for (int s = 0; s < mine; ++s) {
            // all but the RING - 1 stages behind this one have arrived (a pair of scales is among them at the most)
            wait_loads<(RING - 1) * (NLX + NLW) + (MX ? (RING - 1) / 2 * 2 : 0)>();
            const char* tx = ring + from * (XB + WB);
            const char* tw = tx + XB;
            s16x8_t fx[HALVES][FM], fw[HALVES][FN];
            int sx[FM], sw[FN];
            repeat<HALVES>([&](auto h) {
                repeat<FM>([&](auto f) { fx[h.value][f.value] = rx.template get<f.value, h.value>(tx); });
                repeat<FN>([&](auto f) { fw[h.value][f.value] = rw.template get<f.value, h.value>(tw); });
            });
            if constexpr (MX) {
                if ((s & 1) == 0) have ^= 1;
                const char* ts = scales + have * (BM + BN) * 16 + (s & 1) * 8 + q * 2 + i * 16;
                repeat<FM>([&](auto f) { sx[f.value] = *(const uint16_t*)(ts + f.value * 256); });
                repeat<FN>([&](auto f) { sw[f.value] = *(const uint16_t*)(ts + (FM + f.value) * 256); });
            } else {
                repeat<FM>([&](auto f) { sx[f.value] = 0; });
                repeat<FN>([&](auto f) { sw[f.value] = 0; });
            }
            // the fragments are in registers before their place is asked for again
            repeat<HALVES>([&](auto h) {
                repeat<FM>([&](auto f) { hold(fx[h.value][f.value]); });
                repeat<FN>([&](auto f) { hold(fw[h.value][f.value]); });
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const bool turn = ls == mine;
            issue();
            if (turn) {
                next = lt;
                more = at < tiles.end;
            }
            repeat<HALVES>([&](auto h) {
                repeat<FN>([&](auto n) { acc[0][n.value] = multiply<FMT, h.value, h.value>(fw[h.value][n.value], fx[h.value][0], acc[0][n.value], sw[n.value], sx[0]); });
                if constexpr (FM > 1) {
                    if (mrows > 16)
                        repeat<FN>([&](auto n) { acc[1][n.value] = multiply<FMT, h.value, h.value>(fw[h.value][n.value], fx[h.value][1], acc[1][n.value], sw[n.value], sx[1]); });
                }
            });
            from = from == RING - 1 ? 0 : from + 1;
        }

        // partial sums [wave][row][column], the columns of a row in 16-byte chunks turned by the row
        block_barrier();  // (those of the last tile have been read)
        repeat<FM>([&](auto m) {
            repeat<FN>([&](auto n) { *(f32x4_t*)(parts[wave] + (m.value * 16 + i) * BN + ((n.value * 4 + q) ^ (i & 7)) * 4) = acc[m.value][n.value]; });
        });
        block_barrier();
        for (int p = threadIdx.x; p < BM * BN / 8; p += NW * 64) {
            const int row = p / (BN / 8), c = p % (BN / 8);
            if (row >= mrows || c * 8 >= ncols) continue;
            f32x4_t u = {0.f, 0.f, 0.f, 0.f}, v = u;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                u += *(const f32x4_t*)(parts[w] + row * BN + ((2 * c) ^ (row & 7)) * 4);
                v += *(const f32x4_t*)(parts[w] + row * BN + ((2 * c + 1) ^ (row & 7)) * 4);
            }
            if (g.splits > 1) {
                f32x4_t* to = (f32x4_t*)(g.part + t.split * g.slab + (int64_t)(t.lo + t.m0 + row) * g.N + t.n0 + c * 8);
                to[0] = u;
                to[1] = v;
                continue;
            }
            const u32x4_t o = {pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            *(u32x4_t*)((uint16_t*)g.c + (int64_t)(t.lo + t.m0 + row) * g.ldc + t.n0 + c * 8) = o;
        }
        if (!more) break;
        t = next;
    }
    wait_loads<0>();  // nothing may arrive in LDS after the workgroup has left it
}

// A product over ragged rows on the kernel with tiles of bm rows.
template <int FMT, int LB> static inline hipError_t launch_rows(const GroupedArgs& g, int bm, hipStream_t st) {
    if (bm == 16) grouped_stream_kernel<FMT, LB, 16, 3><<<256, 256, 0, st>>>(g);
    else if (bm == 32) grouped_stream_kernel<FMT, LB, 32, 2><<<256, 256, 0, st>>>(g);
    else if (bm == 128) return launch_tiles<FMT, LAY_K, LB, OUT_BF16, 128, 128, 2, 2>(g, st);
    else if constexpr (FMT == FMT_BF16) {
        if (g.part != nullptr) return launch_tiles<FMT, LAY_K, LB, OUT_BF16, 256, 256, 2, 4, true>(g, st);
        return launch_tiles<FMT, LAY_K, LB, OUT_BF16, 256, 256, 2, 4>(g, st);
    } else return launch_tiles<FMT, LAY_K, LB, OUT_BF16, 256, 256, 2, 4>(g, st);
    return hipGetLastError();
}
