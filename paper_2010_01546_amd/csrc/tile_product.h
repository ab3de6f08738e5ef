#pragma once
// Products of two matrices on the matrix cores, for bfloat16 entries (float32 sums) and 8-bit integers (32-bit integer sums), with an
// epilogue of the caller's:  C[r][c] = sum_k A[r][k] B[c][k].
//
// A workgroup owns a tile of 64 NRT x 64 NCT results.  Its wavefronts, two below each other and NW / 2 side by side, hold their parts in
// accumulation registers, as 16 x 16 results of v_mfma_f32_16x16x32_bf16 or v_mfma_i32_16x16x64_i8.  (32 x 32 results need fewer
// instructions and the same operands, but the chip runs them slower under its power limit: random bfloat16 operands in registers, 1.46
// to 1.70 PFLOP/s against 1.91 to 2.08.)  B is the first operand, so that a lane holds four columns next to each other of one row.
// The contraction goes by in stages of 128 bytes of every row of the two panels, so that the loads ask for whole cache lines: a compute
// unit has about 110 requests to its L2 under way, whatever their size, and with 64 bytes each those bound the kernel (loads alone, 8192 x
// 24576 x 4608: 1290 us against 1020).  A ring of stages lies in LDS, filled by loads that go there directly, one barrier per stage.  The
// fragment reads of the next half of a stage and the loads of a later stage are placed between the matrix instructions of this half.
//
// An operand lies in memory in one of two ways.
//   Rows along the contraction (k contiguous): a stage holds 128 bytes of each row, eight chunks of 16; chunk c of row r lies at
//     c ^ (r / 2 % 8), which spreads the 16 rows that are read together over all banks.
//   Contraction-major (bfloat16; a row of memory is one k): a stage holds 64 k of all the panel's columns and is turned as it is read
//     (ds_read_b64_tr_b16: 16 lanes get 4 k of a column each out of 4 x 16 entries).  Pairs of chunks, 16 columns, are permuted by a
//     function of k that puts the eight k read together into different banks.  No transposed copy is made.
// TILE_PLANES: float32 operands as three bfloat16 planes each, x = h + m + l (h = bf16(x), m = bf16(x - h), l = bf16(x - h - m), 24 bits;
//   splitting into three: G. Henry, P. T. P. Tang, A. Heinecke 2019), aplane and bplane bytes apart.  A stage holds all planes of both
//   panels; of their nine products the six above 2^-24 go into the same float32 sums: l h, m h, h h, h m, m m, h l.  (Every pair of planes
//   as a product of its own, each with its loads: 1024 x 576 x 2304, 61 us forward; loads bound it.)  The planes are padded with zeros to
//   whole stages.  Entries below 2^-110 lose their last bits (bfloat16 ends at 2^-133); where a result is not finite (an infinite entry
//   has no such sum) the epilogue computes its 16 x 16 once more in float32.
// Two operands A may meet the same B one after the other (once): sums of a product whose A is the sum of two bfloat16 numbers.
// Where the contraction ends inside a stage, the loads past the end fetch a zero (in both operands: 0 x NaN is NaN).  Rows or columns past
// the edge are clamped; they feed results that the epilogue does not store.
//
// Tiles that do not fill the chip (few tiles, or the rest behind whole rounds of 256): the contraction of these is cut into runs over more
// workgroups, which leave their sums in a workspace, in the order of the accumulation registers; a second launch adds them in order and
// applies the epilogue.
#include "fw_internal.h"
#include <type_traits>

namespace fw {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

static __device__ uint4 tile_zero;          // 16 bytes of zeros, never written

enum TileKind { TILE_BF16, TILE_I8, TILE_PLANES, TILE_F32 };      // TILE_F32: few rows alone

struct TileProduct {
    const char *a, *b0, *b1;      // operands; b1: a second matrix, of the same tile's other columns (PAIR) or of the contraction's second part
    long long apitch, bpitch;     // bytes between rows in memory
    int R, C;                     // results; PAIR: C columns of each matrix
    int chunks;                   // 16-byte chunks of a row (operands along the contraction)
    int klen;                     // k of a part (contraction-major operands)
    int part, once, stages;       // stages of a part, of one pass over B, in all
    long long aplane, bplane;     // TILE_PLANES: bytes between planes; once < stages: aplane to the second operand that meets B again
    int nrb, ncb;                 // rows and columns of tiles
    int full, rest;               // tiles with the whole contraction, tiles cut into runs (none where runs is 1)
    int runs, spr;                // runs, stages of a run
    int nrt, nct;                 // tile shape
    void* partial;
};

// Tiles in bands of eight rows of tiles, column by column inside a band: the 32 tiles that an XCD works on at a time share eight row
// panels and four column panels.
__device__ __forceinline__ void tile_at(const TileProduct& g, int tile, int& I, int& J) {
    const int band = tile / (8 * g.ncb), h = min(8, g.nrb - 8 * band), in = tile - band * 8 * g.ncb;
    J = in / h;
    I = 8 * band + in - J * h;
}

// permutation of the pairs of chunks of row k of a contraction-major panel of 64 N columns
template <int N> __device__ __forceinline__ int pair_swizzle(int k) {
    return N > 1 ? (k & 3) | ((k >> 1) & 4) : ((k >> 1) & 1) | ((k >> 2) & 2);
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// dma16 (fw_internal.h) from an address that is the same for the wavefront plus 32 bits of a lane's own: no vector arithmetic
__device__ __forceinline__ void dma16_from(const void* base, unsigned offset, void* lds_dst) {
    const unsigned lds_addr = (unsigned)(size_t)(__attribute__((address_space(3))) void*)lds_dst;
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(lds_addr) : "memory", "m0");
}
#pragma clang diagnostic pop

template <int I, int N, class F> __device__ __forceinline__ void static_for(const F& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        static_for<I + 1, N>(f);
    }
}

template <int NRT, int NCT, int NW> struct TileShape {
    static constexpr int NWC = NW / 2;                          // wavefronts side by side
    static constexpr int WR = 2 * NRT, WC = 4 * NCT / NWC;      // 16 x 16 results of a wavefront, down and across
    static constexpr int NT = 64 * NW;
    static constexpr int PA = 8192 * NRT, PB = 8192 * NCT;      // bytes of a stage of a panel
    // stages of B in LDS, one more of A: what 160 KB hold
    static constexpr int D = NRT + NCT >= 8 ? 2 : NRT + NCT >= 5 ? 3 : NRT + NCT == 4 ? 4 : 6;
    static_assert((D + 1) * PA + D * PB <= 160 * 1024, "LDS of a compute unit");
};
template <int WC, bool PAIR> __device__ __forceinline__ int tile_column(int panel, int wj, int lane) {
    return panel + wj * (PAIR ? 8 * WC : 16 * WC) + 4 * (lane >> 4);
}
// the finished sums of a wavefront's row of 16 x 16 results: row n, from column s on
template <int WC, bool PAIR, class Acc, class Epi>
__device__ __forceinline__ void tile_apply(const Epi& epi, int n, int s, const Acc (&acc)[WC]) {
#pragma unroll
    for (int tb = 0; tb < (PAIR ? WC / 2 : WC); ++tb) {
        if constexpr (PAIR) epi.apply(n, s + 16 * tb, acc[tb], acc[tb + WC / 2]);
        else epi.apply(n, s + 16 * tb, acc[tb]);
    }
}

// what an epilogue does once a wavefront's results, `rows` from row n and `columns` from column s on, are stored
template <class Epi> __device__ __forceinline__ auto tile_finish(const Epi& epi, int n, int rows, int s, int columns, int) -> decltype(epi.finish(n, rows, s, columns)) {
    epi.finish(n, rows, s, columns);
}
template <class Epi> __device__ __forceinline__ void tile_finish(const Epi&, int, int, int, int, long) {}

// PAIR: the panel of B holds columns of b0 and the same columns of b1; results tb and tb + WC / 2 of a wavefront belong together.
template <TileKind KIND, int NRT, int NCT, int NW, bool AKM, bool BKM, bool PAIR, class Epi>
__global__ __launch_bounds__(64 * NW, 2) void tile_product_kernel(TileProduct g, Epi epi) {
    using Shape = TileShape<NRT, NCT, NW>;
    constexpr bool I8 = KIND == TILE_I8, PLANES = KIND == TILE_PLANES;
    constexpr int D = Shape::D, NWC = Shape::NWC, WR = Shape::WR, WC = Shape::WC;
    constexpr int LA = 8 * NRT / NW, LB = 8 * NCT / NW, NL = LA + LB;      // loads of a wavefront and stage
    constexpr int NF = WR + WC, NM = WR * WC;                             // fragments, matrix instructions
    using Acc = typename std::conditional<I8, intx4, floatx4>::type;
    __shared__ __align__(1024) char lds[PLANES ? 3 * (Shape::PA + Shape::PB) : (D + 1) * Shape::PA + D * Shape::PB];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / NWC, wj = wave % NWC;
    // workgroups go to the 8 XCDs in turn: each XCD gets a contiguous piece of the whole tiles, then one of the runs
    const int items = g.rest * g.runs, per_full = (g.full + 7) / 8, per_run = (items + 7) / 8;
    int at = (int)blockIdx.x >> 3;
    int tile, run = 0, c0 = 0, cend = g.stages;
    const bool cut = at >= per_full;
    if (cut) {
        at += ((int)blockIdx.x & 7) * per_run - per_full;
        if (at >= items) return;
        run = __builtin_amdgcn_readfirstlane(at / g.rest);
        tile = g.full + at - run * g.rest;
        c0 = run * g.spr;
        cend = min(c0 + g.spr, g.stages);
    } else {
        tile = ((int)blockIdx.x & 7) * per_full + at;
        if (tile >= g.full) return;
    }
    int I, J;
    tile_at(g, tile, I, J);
    I = __builtin_amdgcn_readfirstlane(I); J = __builtin_amdgcn_readfirstlane(J);

    // What this lane brings: of each panel a wavefront loads 1 KB pieces wave, wave + NW, ..., from base_a or base_b (the same for the
    // wavefront) + the stage's offset + vof[k]
    const char *base_a, *base_b;
    unsigned vof[NL];
    const int chunk = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));        // rows along the contraction: eight rows a piece, NW is even
    auto along = [&](int row0, int rows, long long pitch, int first, int k) __attribute__((always_inline)) {
        vof[k] = (unsigned)((min(row0 + (lane >> 3), rows - 1) - first) * pitch) + 16 * chunk;
    };
    auto major = [&](auto N, long long pitch, int tile0, int cols, int k, int at) __attribute__((always_inline)) {
        constexpr int CH = 8 * decltype(N)::value, RP = 64 / CH;          // chunks of a row of the panel, rows of a piece
        static_assert(NW * RP % 16 == 0, "the permutation goes by four bits of the row and is the same for all pieces of a lane");
        const int c = (lane % CH) ^ (2 * pair_swizzle<decltype(N)::value>(wave * RP + lane / CH));
        vof[at] = (unsigned)(((wave + NW * k) * RP + lane / CH) * pitch) + 16 * min(tile0 * CH + c, (cols + 7) / 8 - 1);
    };
    if constexpr (AKM) {
        base_a = g.a;
#pragma unroll
        for (int k = 0; k < LA; ++k) major(std::integral_constant<int, NRT>(), g.apitch, I, g.R, k, k);
    } else {
        const int first = I * 64 * NRT;
        base_a = g.a + first * g.apitch;
#pragma unroll
        for (int k = 0; k < LA; ++k) along(first + 8 * (wave + NW * k), g.R, g.apitch, first, k);
    }
    if constexpr (BKM) {
        base_b = g.b0;
#pragma unroll
        for (int k = 0; k < LB; ++k) major(std::integral_constant<int, NCT>(), g.bpitch, J, g.C, k, LA + k);
    } else {
        const int first = J * (PAIR ? 32 : 64) * NCT;
        const int w = 8 * wave % (16 * WC);                              // place in the wavefront's part of the panel, the same for all pieces
        static_assert(!PAIR || 8 * NW % (16 * WC) == 0, "a wavefront brings columns of one matrix");
        base_b = (PAIR && w >= 8 * WC ? g.b1 : g.b0) + first * g.bpitch;
#pragma unroll
        for (int k = 0; k < LB; ++k) {
            const int pr = 8 * (wave + NW * k);
            along(first + (PAIR ? pr / (16 * WC) * 8 * WC + w % (8 * WC) : pr), g.C, g.bpitch, first, LA + k);
        }
    }
    const long long second = BKM ? g.b1 - g.b0 : 0;
    // stages that lie inside the contraction with all their chunks (of a part)
    const int whole = AKM || BKM ? g.klen >> 6 : g.chunks >> 3;
    struct Stage { const char *a, *b; int c, ca, cb; };         // stage, and within a pass over B and a part
    auto stage_at = [&](int c) __attribute__((always_inline)) {
        Stage s;
        s.c = c;
        const bool again = BKM && KIND == TILE_BF16 && c >= g.once;
        s.ca = again ? c - g.once : c;
        const bool two = BKM && s.ca >= g.part;
        s.cb = two ? s.ca - g.part : s.ca;
        s.a = base_a + (AKM ? (long long)s.ca * 64 * g.apitch : (long long)s.ca * 128) + (again ? g.aplane : 0);
        s.b = base_b + (BKM ? (long long)s.cb * 64 * g.bpitch + (two ? second : 0) : (long long)c * 128);
        return s;
    };
    // ALL: the whole stage lies inside the contraction
    auto load_one = [&](auto ALL, int to_buf, const Stage& s, int k) __attribute__((always_inline)) {      // k is a constant after unrolling
        const bool isa = k < LA;
        void* to = &lds[to_buf + 1024 * (wave + NW * (isa ? k : k - LA))];
        if constexpr (decltype(ALL)::value) {
            dma16_from(isa ? s.a : s.b, vof[k], to);
        } else {
            const int c = isa ? s.ca : s.cb, RP = 8 / (isa ? NRT : NCT);
            const bool major = isa ? AKM : BKM;
            const bool inside = s.c < cend && (major ? 64 * c + (wave + NW * (isa ? k : k - LA)) * RP + lane / (64 / RP) < g.klen
                                                     : 8 * c + chunk < g.chunks);
            dma16(inside ? (const void*)((isa ? s.a : s.b) + vof[k]) : (const void*)&tile_zero, to);
        }
    };

    Acc acc[WR][WC];
#pragma unroll
    for (int a = 0; a < WR; ++a)
#pragma unroll
        for (int b = 0; b < WC; ++b) acc[a][b] = Acc{0, 0, 0, 0};

    // Fragment f of half h of a stage: 16 rows of A, then of B.  Where a lane reads: its own place, with 64 h flipped in and + 2048 f for
    // rows along the contraction, with 32 f flipped in and 32 rows further on for the second half of a contraction-major panel (the
    // permutations touch only those bits).
    intx4 fr[2][NF];
    const int l16 = lane & 15, q = lane >> 4, kq = 8 * q + (l16 >> 2);       // kq + 4 and kq + 32 have the permutation of kq
    const int along_at = l16 * 128 + 16 * (q ^ (l16 >> 1));
    const int at_a = AKM ? kq * 128 * NRT + 32 * (wi * WR ^ pair_swizzle<NRT>(kq)) + 8 * (l16 & 3) : wi * WR * 2048 + along_at;
    const int at_b = (BKM ? kq * 128 * NCT + 32 * (wj * WC ^ pair_swizzle<NCT>(kq)) + 8 * (l16 & 3) : wj * WC * 2048 + along_at);
    auto read_one = [&](int a, int b, int half, int f) __attribute__((always_inline)) {    // a, b: at_a and at_b in the stage's buffers
        const bool isa = f < WR;
        const int r = isa ? f : f - WR;
        const char* all = lds;
        if (isa ? AKM : BKM) {
            const int rowb = 128 * (isa ? NRT : NCT);
            const char* p = all + ((isa ? a : b) ^ (32 * r)) + 32 * half * rowb;
            typedef __attribute__((address_space(3))) shortx4* lp;
            union { shortx4 h[2]; intx4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * rowb));
            fr[half][f] = u.v;
        } else {
            fr[half][f] = *reinterpret_cast<const intx4*>(all + ((isa ? a : b) ^ (64 * half)) + 2048 * r);
        }
    };
    auto multiply_one = [&](int half, int m) __attribute__((always_inline)) {
        const int ta = m / WC, tb = m % WC;
        if constexpr (I8)
            acc[ta][tb] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fr[half][WR + tb], fr[half][ta], acc[ta][tb], 0, 0, 0);
        else
            acc[ta][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fr[half][WR + tb]),
                                                                  __builtin_bit_cast(bf16x8, fr[half][ta]), acc[ta][tb], 0, 0, 0);
    };

    // The reads go over the first three quarters of the matrix instructions (the last ones have to be back when the next half begins).
    // LOADS: 0 none, 1 a panel of A, 2 of B.
    auto half_turn = [&](int ra, int rb, auto HALF, auto LOADS, auto ALL, int to_buf, const Stage& next) __attribute__((always_inline)) {
        constexpr int half = decltype(HALF)::value, what = decltype(LOADS)::value;
        constexpr int K0 = what == 1 ? 0 : LA, KN = what == 0 ? 0 : what == 1 ? LA : LB;
        static_for<0, NM>([&](auto M) __attribute__((always_inline)) {
            constexpr int m = decltype(M)::value;
#pragma unroll
            for (int r = 0; r < NF; ++r)
                if (r * (3 * NM) / (4 * NF) == m) read_one(ra, rb, half ^ 1, r);
#pragma unroll
            for (int k = 0; k < KN; ++k)
                if (k * NM / (KN ? KN : 1) + (NM > KN) == m) load_one(ALL, to_buf, next, K0 + k);
            multiply_one(half, m);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    if constexpr (!PLANES) {
        // At the barrier in the middle of stage c every wavefront holds the stage's second half in registers, so its buffers are free: in the
        // half that follows the loads of B's stage c + D go out, in the half after that those of A's stage c + D + 1.  The loads of a wavefront
        // complete in order; with those behind B's stage c + 1 outstanding all of that stage has landed for it, the barrier extends that to
        // all.  Past the end the loads fetch zeros, which keeps their number the same.  (Small tiles gain from a deep ring: 501 x 2304 x
        // 6145, two projections, 39.7 us with two stages of B, 36.6 with three.)
        auto load_panel = [&](auto ISA, int to_buf, int c) __attribute__((always_inline)) {
            const Stage s = stage_at(c);
#pragma unroll
            for (int k = decltype(ISA)::value ? 0 : LA; k < (decltype(ISA)::value ? LA : NL); ++k) load_one(std::false_type(), to_buf, s, k);
        };
        constexpr int B0 = (D + 1) * Shape::PA, BE = B0 + D * Shape::PB;
        for (int i = 0; i < D; ++i) {
            load_panel(std::true_type(), i * Shape::PA, c0 + i);
            load_panel(std::false_type(), B0 + i * Shape::PB, c0 + i);
        }
        FW_WAIT_VM((D - 1) * NL);
        __builtin_amdgcn_s_barrier();
        FW_COMPILER_FENCE();
#pragma unroll
        for (int f = 0; f < NF; ++f) read_one(at_a, B0 + at_b, 0, f);
        int a0 = 0, b0 = B0;                         // the stage's buffers
        int c = c0, begun = 0;                       // the part that stage c + D lies in
        auto turn = [&](auto ALL) __attribute__((always_inline)) {
            const int a1 = a0 == D * Shape::PA ? 0 : a0 + Shape::PA, free_a = a0 == 0 ? D * Shape::PA : a0 - Shape::PA;
            const int b1 = b0 == BE - Shape::PB ? B0 : b0 + Shape::PB;
            const Stage next = stage_at(c + D);
            half_turn(at_a + a0, at_b + b0, std::integral_constant<int, 0>(), std::integral_constant<int, 1>(), ALL, free_a, next);
            FW_WAIT_LGKM0();
            FW_WAIT_VM((D - 1) * LA + (D - 2) * LB);
            __builtin_amdgcn_s_barrier();
            FW_COMPILER_FENCE();
            half_turn(at_a + a1, at_b + b1, std::integral_constant<int, 1>(), std::integral_constant<int, 2>(), ALL, b0, next);
            a0 = a1; b0 = b1;
            ++c;
        };
        while (c < cend) {
            // stages up to `fast` ask for whole ones only
            while (BKM && c + D >= begun + g.part) begun += g.part;
            const int fast = min(cend, begun + min(whole, g.part)) - D;
            while (c < fast) turn(std::true_type());
            turn(std::false_type());
        }
    } else {
        // A panel of the next stage is asked for when its plane was used last in this one, over two halves where two planes end
        // together.  vmcnt: what may be outstanding is what was asked for behind the panel that the next product needs.
        using std::integral_constant;
        constexpr integral_constant<int, 0> H0, NONE;
        constexpr integral_constant<int, 1> H1, PANEL_A;
        constexpr integral_constant<int, 2> PANEL_B;
        constexpr std::true_type ALL;
        constexpr int AH = 0, AM = Shape::PA, AL = 2 * Shape::PA, BH = 3 * Shape::PA, BM = BH + Shape::PB, BL = BM + Shape::PB;
        auto plane = [&](Stage s, int p) __attribute__((always_inline)) { s.a += p * g.aplane; s.b += p * g.bplane; return s; };     // 0 h, 1 m, 2 l
        auto load_panel = [&](auto A, int buf, const Stage& s) __attribute__((always_inline)) {
#pragma unroll
            for (int k = decltype(A)::value ? 0 : LA; k < (decltype(A)::value ? LA : NL); ++k) load_one(ALL, buf, s, k);
        };
        const Stage first = stage_at(c0);
        load_panel(std::true_type(), AL, plane(first, 2));
        load_panel(std::false_type(), BH, first);
        load_panel(std::true_type(), AM, plane(first, 1));
        load_panel(std::false_type(), BM, plane(first, 1));
        load_panel(std::true_type(), AH, first);
        load_panel(std::false_type(), BL, plane(first, 2));
        auto meet = [&](auto VM) __attribute__((always_inline)) {
            FW_WAIT_LGKM0();
            FW_WAIT_VM(decltype(VM)::value);
            __builtin_amdgcn_s_barrier();
            FW_COMPILER_FENCE();
        };
        meet(integral_constant<int, 2 * LA + 2 * LB>());
#pragma unroll
        for (int f = 0; f < NF; ++f) read_one(at_a + AL, at_b + BH, 0, f);
        Stage now = first;
        for (int c = c0; c < cend; ++c) {
            const Stage next = stage_at(min(c + 1, cend - 1));       // past the end the last stage once more, unread
            half_turn(at_a + AL, at_b + BH, H0, PANEL_B, ALL, BL, plane(now, 2));             // l h; the loads are of this stage (see below)
            meet(integral_constant<int, LA + 2 * LB>());                                      // m
            half_turn(at_a + AM, at_b + BH, H1, PANEL_A, ALL, AL, plane(next, 2));
            half_turn(at_a + AM, at_b + BH, H0, NONE, ALL, 0, next);                          // m h
            meet(integral_constant<int, LA + LB>());                                          // h of A
            half_turn(at_a + AH, at_b + BH, H1, NONE, ALL, 0, next);
            half_turn(at_a + AH, at_b + BH, H0, NONE, ALL, 0, next);                          // h h
            meet(integral_constant<int, LA + LB>());                                          // (m of B is older than h of A)
            half_turn(at_a + AH, at_b + BM, H1, PANEL_B, ALL, BH, next);
            half_turn(at_a + AH, at_b + BM, H0, NONE, ALL, 0, next);                          // h m
            FW_WAIT_LGKM0();
            half_turn(at_a + AM, at_b + BM, H1, NONE, ALL, 0, next);
            half_turn(at_a + AM, at_b + BM, H0, NONE, ALL, 0, next);                          // m m
            meet(integral_constant<int, LA + LB>());                                          // l of B
            half_turn(at_a + AH, at_b + BL, H1, PANEL_A, ALL, AM, plane(next, 1));
            half_turn(at_a + AH, at_b + BL, H0, PANEL_B, ALL, BM, plane(next, 1));            // h l
            meet(integral_constant<int, LA + LB>());                                          // the next stage's l of A and h of B
            half_turn(at_a + AL, at_b + BH, H1, PANEL_A, ALL, AH, next);
            now = next;
        }
    }
    FW_WAIT_VM(0);
    FW_WAIT_LGKM0();

    if (cut) {
        Acc* out = reinterpret_cast<Acc*>(g.partial) + ((size_t)run * g.rest + tile - g.full) * (NM * Shape::NT) + tid;
#pragma unroll
        for (int ta = 0; ta < WR; ++ta)
#pragma unroll
            for (int tb = 0; tb < WC; ++tb) out[(ta * WC + tb) * Shape::NT] = acc[ta][tb];
        return;
    }
    const int s = tile_column<WC, PAIR>(J * (PAIR ? 32 : 64) * NCT, wj, lane);
#pragma unroll
    for (int ta = 0; ta < WR; ++ta) tile_apply<WC, PAIR>(epi, I * 64 * NRT + 16 * (wi * WR + ta) + l16, s, acc[ta]);
    tile_finish(epi, I * 64 * NRT + 16 * wi * WR, 16 * WR, s - 4 * q, 16 * WC, 0);
}

// adds the runs of a tile's rows of 16 x 16 results, in order, and applies the epilogue
template <bool I8, int NRT, int NCT, int NW, bool PAIR, class Epi>
__global__ __launch_bounds__(64 * NW) void tile_runs_kernel(TileProduct g, Epi epi) {
    using Shape = TileShape<NRT, NCT, NW>;
    constexpr int WR = Shape::WR, WC = Shape::WC;
    using Acc = typename std::conditional<I8, intx4, floatx4>::type;
    const int tile = blockIdx.x / WR, ta = blockIdx.x % WR;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wi = wave / Shape::NWC, wj = wave % Shape::NWC;
    int I, J;
    tile_at(g, g.full + tile, I, J);
    Acc acc[WC];
    const Acc* in = reinterpret_cast<const Acc*>(g.partial) + ((size_t)tile * WR + ta) * (WC * Shape::NT) + tid;
#pragma unroll
    for (int tb = 0; tb < WC; ++tb) acc[tb] = in[tb * Shape::NT];
    for (int z = 1; z < g.runs; ++z) {
        in += (size_t)g.rest * (WR * WC * Shape::NT);
#pragma unroll
        for (int tb = 0; tb < WC; ++tb) {
            const Acc v = in[tb * Shape::NT];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[tb][i] += v[i];
        }
    }
    const int n = I * 64 * NRT + 16 * (wi * WR + ta), s = tile_column<WC, PAIR>(J * (PAIR ? 32 : 64) * NCT, wj, lane);
    tile_apply<WC, PAIR>(epi, n + (lane & 15), s, acc);
    tile_finish(epi, n, 16, s - 4 * (lane >> 4), 16 * WC, 0);
}

// ---- what the epilogues store: four entries of a row from column s on, of `cols`
__device__ __forceinline__ void tile_store(__bf16* p, int s, int cols, const float (&v)[4]) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    if (s + 4 <= cols) {
        const bf16x4 o = {(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        __builtin_memcpy(p, &o, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (s + i < cols) p[i] = (__bf16)v[i];
    }
}
__device__ __forceinline__ void tile_store(float* p, int s, int cols, const float (&v)[4]) {
    if (s + 4 <= cols) {
        __builtin_memcpy(p, v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (s + i < cols) p[i] = v[i];
    }
}
// four entries of a vector from column s on, zero beyond the end and for no vector
__device__ __forceinline__ void tile_vector(const float* p, int s, int cols, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = p && s + i < cols ? p[s + i] : 0.f;
}

// Tile shape and runs of the least estimated time in cycles (2.1 GHz): rounds of 256 workgroups x (stages x the longer of a stage's matrix
// instructions and its loads + the first loads + storing the results, `bytes` each), plus the launch that adds the runs and its traffic.
// Runs are for the tiles behind whole rounds, and keep at least 4 stages (of planes: 2, each with six products).
// The constants are fitted to 123 products (20 to 8192 rows, 64 to 12288 columns and features) with every shape and number of runs
// measured: what is chosen takes 0.5 % longer than the best on average, 8 % at most.  The projections among them stored Z; without it they
// are planned alike, though they store a third to a fifth (501 x 2304 x 6145: 42 us without, 52 with).
// even: an even number of 64 rows (both weights' gradients below each other), of which 64 x 256 results never beat 128 x 128: as many
// tiles or more, longer loads.
inline void tile_plan(TileProduct& g, bool pair, bool planes, double bytes, bool even = false) {
    static const int shapes[][2] = {{4, 4}, {2, 4}, {2, 2}, {1, 4}, {1, 2}};
    double best = 1e300;
    for (int i = planes ? 1 : 0; i < 5; ++i) {               // the planes of 256 x 256 results do not fit into LDS
        if (even && i == 3) continue;
        const int nrt = shapes[i][0], nct = shapes[i][1], tc = pair ? 32 * nct : 64 * nct;
        const int nrb = (g.R + 64 * nrt - 1) / (64 * nrt), ncb = (g.C + tc - 1) / tc;
        const long long tiles = (long long)nrb * ncb;
        const double area = nrt * nct, t_mfma = (planes ? 6 * 130.0 : 145.0) * area + 60.0, t_load = (nrt + nct) * 8192.0 / 30.0 * (planes ? 3 : 1);
        const double t_stage = t_mfma > t_load ? t_mfma : t_load, fill = 2150.0, store = 1250.0 * bytes * area;
        const int rest = (int)(tiles % 256);
        for (int runs = 1; runs <= 32 && (runs == 1 || (rest > 0 && rest * runs <= 512 && g.stages / runs >= (planes ? 2 : 4))); ++runs) {
            const int spr = (g.stages + runs - 1) / runs, n = (g.stages + spr - 1) / spr;
            double cost = (double)((n > 1 ? tiles : tiles + 255) / 256) * (g.stages * t_stage + fill + store);
            if (n > 1)
                cost += (double)((rest * n + 255) / 256) * (spr * t_stage + fill) + rest / 256.0 * store + 9500.0 +
                        2.0 * n * rest * (area * 16384.0) / 4.1e12 * 2.1e9;
            if (cost < best * 0.999) {
                best = cost;
                g.nrt = nrt; g.nct = nct; g.nrb = nrb; g.ncb = ncb; g.runs = n; g.spr = spr;
                g.rest = n > 1 ? rest : 0; g.full = (int)tiles - g.rest;
            }
        }
    }
}
inline TileChoice tile_choice(const TileProduct& g, bool pair) {
    return {0, 64 * g.nrt, (pair ? 32 : 64) * g.nct, g.full, g.rest, g.runs, g.stages};
}
inline size_t tile_partial_bytes(const TileProduct& g) { return align_up((size_t)g.rest * g.runs * g.nrt * g.nct * 16384, 256); }

template <TileKind KIND, int NRT, int NCT, int NW, bool AKM, bool BKM, bool PAIR, class Epi>
fw_status tile_launch(const TileProduct& g, const Epi& epi, hipStream_t st) {
    if ((long long)g.nrb * g.ncb > (1 << 28)) return FW_ERR_UNSUPPORTED;
    const unsigned groups = 8u * (unsigned)((g.full + 7) / 8 + (g.rest * g.runs + 7) / 8);
    hipLaunchKernelGGL((tile_product_kernel<KIND, NRT, NCT, NW, AKM, BKM, PAIR, Epi>), dim3(groups), dim3(64 * NW), 0, st, g, epi);
    FW_LAUNCH_CHECK();
    if (g.rest) {
        hipLaunchKernelGGL((tile_runs_kernel<KIND == TILE_I8, NRT, NCT, NW, PAIR, Epi>), dim3((unsigned)(g.rest * 2 * NRT)), dim3(64 * NW), 0, st, g, epi);
        FW_LAUNCH_CHECK();
    }
    return FW_OK;
}

template <TileKind KIND, bool AKM, bool BKM, bool PAIR, class Epi>
fw_status tile_product(const TileProduct& g, const Epi& epi, hipStream_t st) {
    if constexpr (KIND != TILE_PLANES)
        if (g.nrt == 4) return tile_launch<KIND, 4, 4, 8, AKM, BKM, PAIR>(g, epi, st);
    if (g.nrt == 2 && g.nct == 4) return tile_launch<KIND, 2, 4, 8, AKM, BKM, PAIR>(g, epi, st);
    if (g.nrt == 2) return tile_launch<KIND, 2, 2, 8, AKM, BKM, PAIR>(g, epi, st);
    if constexpr (!AKM)                                      // the rows are outputs of both weights: an even number of 64 (tile_plan)
        if (g.nct == 4) return tile_launch<KIND, 1, 4, 8, AKM, BKM, PAIR>(g, epi, st);
    return tile_launch<KIND, 1, 2, 8, AKM, BKM, PAIR>(g, epi, st);
}

// ---- few rows: C[r][c] = sum_k A[r][k] B[c][k] for up to 16 NA rows, rows along the contraction and of any length.  Bound by
// the one read of B; float32 (products by v_mfma_f32_16x16x4_f32) from about 50 rows on by the matrix instructions.
// A workgroup owns `cols` columns (PAIR: of each matrix), so many that every compute unit gets as much of B to read; its wavefronts take
// stages of 128 bytes in turn, two ahead in registers, turn them through LDS of their own (eight lanes load the 128 bytes of a
// row, so that whole cache lines are asked for) and add up their sums at the end: one launch, no workspace, no padded copies.
// Two projections of one row of 4608 bfloat16, 12288 columns: 39 us, 5.8 TB/s; 16 rows of 12288 bytes, 4608 columns: 14.7 us, 3.8 TB/s.
// (Back to back, which leaves smaller weights in the last-level cache, 42.7 and 11.6 us, tiles of 64 rows whose contraction is cut into
// runs 43.7 and 18.0; 1 x 1153, 1001 columns, whose rows these need padded: 13.3
// against 5.9.)
struct FewProduct {
    const char *a, *b0, *b1;
    int N, C, bytes, cols;        // rows, columns (PAIR: of each matrix), bytes of a row, columns of a workgroup
};
template <TileKind KIND, int NA, bool PAIR, class Epi>
__global__ __launch_bounds__(512, NA > 1 ? 2 : 4) void few_product_kernel(FewProduct g, Epi epi) {
    constexpr bool I8 = KIND == TILE_I8;
    constexpr int NW = 8, NV = 4 + 2 * NA;                            // pieces of 8 rows of a stage: 32 rows of B, 16 NA of A
    using Acc = typename std::conditional<I8, intx4, floatx4>::type;
    __shared__ __align__(16) char lds[NW][1024 * NV];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col0 = blockIdx.x * g.cols, cend = min(g.C, col0 + g.cols);
    const int chunks = g.bytes / 16, stages = (g.bytes + 127) / 128;       // whole chunks of 16 bytes
    // where the rows of a stage begin, behind addresses that are the same for the workgroup
    const char *b0 = g.b0 + (size_t)col0 * g.bytes, *b1 = (PAIR ? g.b1 : g.b0) + (size_t)col0 * g.bytes;
    unsigned at[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int r = 8 * j + (lane >> 3);
        at[j] = (unsigned)(j < 4 ? min(PAIR ? r & 15 : r, cend - 1 - col0) : min(r - 32, g.N - 1)) * g.bytes;
    }
    auto base = [&](int j) __attribute__((always_inline)) { return j < 2 ? b0 : j < 4 ? b1 : g.a; };
    struct Stage { intx4 v[NV]; };
    auto load = [&](Stage& s, int c) __attribute__((always_inline)) {       // chunks outside of the rows: zeros
        const bool in = c >= 0 && 8 * c + (lane & 7) < chunks;
#pragma unroll
        for (int j = 0; j < NV; ++j) __builtin_memcpy(&s.v[j], in ? base(j) + at[j] + 128 * c + 16 * (lane & 7) : reinterpret_cast<const char*>(&tile_zero), 16);
    };
    auto load_whole = [&](Stage& s, int c) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) __builtin_memcpy(&s.v[j], base(j) + 128 * c + (at[j] + 16 * (lane & 7)), 16);
    };
    Acc acc[NA][2];
#pragma unroll
    for (int a = 0; a < NA; ++a) acc[a][0] = acc[a][1] = Acc{0, 0, 0, 0};
    // chunk c of row r at c ^ (r / 2 % 8).  A wavefront's accesses to LDS happen in their order; the fences keep the compiler to it.
    auto use = [&](const Stage& s) __attribute__((always_inline)) {
        FW_COMPILER_FENCE();
#pragma unroll
        for (int j = 0; j < NV; ++j)
            *reinterpret_cast<intx4*>(&lds[wave][(8 * j + (lane >> 3)) * 128 + 16 * ((lane & 7) ^ ((4 * j + (lane >> 4)) & 7))]) = s.v[j];
        FW_COMPILER_FENCE();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            intx4 fr[2 + NA];
#pragma unroll
            for (int f = 0; f < 2 + NA; ++f) fr[f] = *reinterpret_cast<const intx4*>(&lds[wave][(16 * f + l16) * 128 + 16 * ((4 * h + q) ^ (l16 >> 1))]);
#pragma unroll
            for (int m = 0; m < 2 * NA; ++m) {
                const int a = m / 2, f = m % 2;
                if constexpr (I8) {
                    acc[a][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fr[f], fr[2 + a], acc[a][f], 0, 0, 0);
                } else if constexpr (KIND == TILE_BF16) {
                    acc[a][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fr[f]), __builtin_bit_cast(bf16x8, fr[2 + a]), acc[a][f], 0, 0, 0);
                } else {                                       // k = 4 q + i, the same for both operands
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[a][f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(fr[f][i]), __int_as_float(fr[2 + a][i]), acc[a][f], 0, 0, 0);
                }
            }
        }
    };
    Stage s, t;
    int c = stages - 1 - wave, more = c >= 0 ? c / NW - 1 : 0;       // stages behind the first two
    load(s, c);
    if (g.bytes % 16 && wave == 0) {                // the chunk that is not whole
        const int n = 8 * c + (lane & 7) == chunks ? g.bytes - 16 * chunks : 0;
        constexpr int E = I8 ? 1 : KIND == TILE_BF16 ? 2 : 4;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            union { char b[16]; intx4 v; } u;
            u.v = s.v[j];
#pragma unroll
            for (int i = 0; i < 16; i += E)
                if (i < n) __builtin_memcpy(u.b + i, base(j) + at[j] + 16 * chunks + i, E);
            s.v[j] = u.v;
        }
    }
    load(t, c - NW);
    for (c -= 2 * NW; more >= 2; more -= 2, c -= 2 * NW) {
        use(s);
        load_whole(s, c);
        use(t);
        load_whole(t, c - NW);
    }
    use(s);
    if (more == 1) load_whole(s, c);
    use(t);
    if (more == 1) use(s);
    // the wavefronts' sums, in order, 16 rows at a time
#pragma unroll
    for (int a = 0; a < NA; ++a) {
        FW_COMPILER_FENCE();
        if (a) __syncthreads();
#pragma unroll
        for (int f = 0; f < 2; ++f) *reinterpret_cast<Acc*>(&lds[wave][1024 * f + 16 * lane]) = acc[a][f];
        __syncthreads();
        const auto total = [&](int f) __attribute__((always_inline)) {
            Acc v = *reinterpret_cast<const Acc*>(&lds[0][1024 * f + 16 * lane]);
#pragma unroll
            for (int w = 1; w < NW; ++w) {
                const Acc x = *reinterpret_cast<const Acc*>(&lds[w][1024 * f + 16 * lane]);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += x[i];
            }
            return v;
        };
        const int n = 16 * a + l16;
        if constexpr (PAIR) {
            if (wave == 0 && col0 + 4 * q < cend) epi.apply(n, col0 + 4 * q, total(0), total(1));
        } else {
            if (wave < 2 && col0 + 16 * wave + 4 * q < cend) epi.apply(n, col0 + 16 * wave + 4 * q, total(wave));
        }
    }
}
constexpr int few_most(bool pair) { return pair ? 16 : 32; }         // columns a workgroup can take
// bfloat16 and 8 bits: few_product up to 16 rows; up to 64 where there are columns for every compute unit and, if the rows are aligned, not so
// many that a unit takes them in several goes, each with its loads of A.  Tiles against this: projections of 32 rows, 1153 to 4001: 20.6 us and
// 8.9, 2304 to 6145: 16.6 and 13.3, 4608 to 12288: 45.0 and 47.8, 64 to 200: 4.3 and 5.0; of 64 rows, 576 to 2304: 8.5 and 7.3, 2304 to 6145: 17.0
// and 21.3, 2305 to 6145: 41 and 29; 8 bits, 64 rows, 4608 to 4608: 13.7 and 10.8, to 12288: 17.3 and 20.5.
inline bool few_rows(int N, int C, bool aligned, bool pair) {
    return N <= 16 || (N <= 64 && C >= 256 && (!aligned || C <= 256 * few_most(pair) * (N <= 32 ? 2 : 1)));
}
template <TileKind KIND, bool PAIR, int NA, class Epi>
fw_status few_launch(FewProduct g, const Epi& epi, hipStream_t st) {
    const int each = (g.C + 255) / 256, parts = (each + few_most(PAIR) - 1) / few_most(PAIR);
    g.cols = ((each + parts - 1) / parts + 3) / 4 * 4;
    hipLaunchKernelGGL((few_product_kernel<KIND, NA, PAIR, Epi>), dim3((g.C + g.cols - 1) / g.cols), dim3(512), 0, st, g, epi);
    FW_LAUNCH_CHECK();
    return FW_OK;
}

template <TileKind KIND, bool PAIR, class Epi>
fw_status few_product(const FewProduct& g, const Epi& epi, hipStream_t st) {
    if (g.N <= 16) return few_launch<KIND, PAIR, 1>(g, epi, st);
    if (g.N <= 32) return few_launch<KIND, PAIR, 2>(g, epi, st);
    return few_launch<KIND, PAIR, 4>(g, epi, st);
}

}  // namespace fw
